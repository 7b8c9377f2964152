// Windowed attention of blocks of queries on the tensor cores (bf16; e4m3 widened to fp16), and the weights that it gives to the cached rows.
//
// attend_tile_kernel.  A CTA has NT tiles of 128 query rows that share a key head (row r of a tile: query r / g, head r % g of the g heads
// packed side by side, one TMA box) and walks the tiles of BN keys that some of its rows may see:
//     S = Q K^T (tcgen05, both from shared memory)  ->  P = 2^(S - reference), rounded to 16 bits, back into the columns of S
//     ->  O += P V (tcgen05, P from tensor memory, V as it lies in the cache: its rows are the contraction).
// Warps 0-3 and 4-7: the softmax of one tile each, a thread per row: maximum and sum without a shuffle.  The sums in O are taken
// against a reference that is moved only when a row's maximum grows past it by 2^8 (the result is the same; moving it is a pass over O).
// Warp 8 loads, warp 9 issues the MMAs.  Two tiles keep the tensor cores and the exponentials busy in turn; heads above 128 elements
// leave tensor memory for one tile, whose S is double-buffered instead.
// Which key tiles, which of them some row of a tile sees, and which need their mask element by element, is settled before
// the walk, from the positions; rows that nobody may look at have their values set to zero in shared memory (0 times NaN is NaN).
#include "attend.cuh"
#include "tmem_ld.cuh"
#include "tmem_plan.h"
#include "tmem_st.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 320;
constexpr int kRows = 128;                   // query rows of a tile
constexpr int kMaxStages = 6;
constexpr float kMoveAt = 8.f;               // a row's maximum may lie this far (powers of two) above its reference

// D[tmem] (+)= A[tmem] * B[smem], bf16, fp32 accumulate; issued by one thread.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// Shared-memory matrix descriptor of a tile whose rows (128 bytes, 128-byte swizzle) are the contraction: 64 elements of the other
// dimension lie in a row, the next 64 `box` bytes further on, the next 8 rows 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_rows_sw128(uint32_t addr, uint32_t box)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(box >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
// Instruction descriptor of fp16 or bf16 operands (format codes 0 and 1 of both), M = 128, N = n.
template <bool F16>
__device__ __forceinline__ uint32_t idesc_16(int n) { return F16 ? idesc_bf16_m128(n) & ~((1u << 7) | (1u << 10)) : idesc_bf16_m128(n); }
constexpr uint32_t kRowsAreContraction = 1u << 16;      // instruction descriptor: B as above

// Two neighbouring values of a 16-bit type: bf16, and for what came from e4m3 (exactly) fp16, whose weights are finer.
__device__ __forceinline__ uint32_t two_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x)
{
    *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
}

// The lowest n of 32 bits (all of them from 32 on, none below 1).
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }

// An entry of the list of key (or query) tiles that a CTA walks: which of the range, and what has to be done with it.
constexpr int kNeed = 1, kMask = 4, kHidden = 16, kEntryShift = 5;      // kNeed, kMask: shifted by the tile of rows
__device__ __forceinline__ int entry_of(int rel, int flags) { return rel << kEntryShift | flags; }

// Positions of `n` keys from row j0 on, by one warp: smallest and largest of those somebody may see, and whether there are others.
struct Span {
    int lo, hi;
    bool hidden;
};
__device__ __forceinline__ Span key_span(const AttArgs& a, const AttSeq& s, int len, int j0, int n, int lane)
{
    int lo = 0x7FFFFFFF, hi = -1;
    bool hidden = false;
    for (int e = lane; e < n; e += 32) {
        const int c = key_pos(a, s, len, j0 + e);
        if (c < 0) hidden = true;
        else { lo = min(lo, c); hi = max(hi, c); }
    }
    return {__reduce_min_sync(0xffffffffu, lo), __reduce_max_sync(0xffffffffu, hi), __any_sync(0xffffffffu, hidden)};
}
__device__ __forceinline__ Span counted_span(int len, int j0, int n)
{
    return {j0 < len ? j0 : 0x7FFFFFFF, j0 < len ? min(j0 + n, len) - 1 : -1, j0 + n > len};
}
// Whether rows with positions in [lo, hi] see something of a span, and whether all of them see all of it.
__device__ __forceinline__ int span_flags(const AttArgs& a, int lo, int hi, const Span& k)
{
    if (k.hi < 0 || k.lo > hi || !(k.hi >= lo || lo - k.hi < a.window || k.lo < a.n_sink)) return 0;
    const bool all = k.hi <= lo && !k.hidden && (hi - k.lo < a.window || k.hi < a.n_sink);
    return all ? kNeed : kNeed | kMask;
}
// The entries with a flag among `n` flag words, in order, in place; by one warp.  Returns how many.
__device__ __forceinline__ int compact_entries(uint16_t* list, int n, int lane)
{
    int count = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int f = i0 + lane < n ? list[i0 + lane] : 0;
        const unsigned on = __ballot_sync(0xffffffffu, (f & 3) != 0);
        __syncwarp();
        if (f & 3) list[count + __popc(on & ((1u << lane) - 1u))] = static_cast<uint16_t>(entry_of(i0 + lane, f));
        __syncwarp();
        count += __popc(on);
    }
    return count;
}

// Bounded waits of a CTA: when one runs out, the others end without waiting for long.
struct Guard {
    int* dead;
    int* status;
    // by a whole warp: the same answer in all its lanes
    __device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)); }
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity)
    {
        if (mbar_try_wait<false>(bar, parity)) return true;
        if (*reinterpret_cast<volatile int*>(dead)) return false;
        // (the clock of the multiprocessor, about a second of it; the global timer takes a microsecond to read)
        const long long t0 = clock64();
        for (uint32_t it = 1; it < kSpinLimit; ++it) {
            if (mbar_try_wait<false>(bar, parity)) return true;
            if ((it & 63u) == 0 && clock64() - t0 > 2000000000ll) break;
        }
        *reinterpret_cast<volatile int*>(dead) = 1;
        *reinterpret_cast<volatile int*>(status) = MVLA_ERR_TIMEOUT;
        return false;
    }
};

template <int DB, int NT, int BN>
struct TileShape {
    static constexpr int kQBytes = DB * kRows * 128;         // one tile of query rows
    static constexpr int kStage = DB * BN * 128;             // one tile of keys or values
    static constexpr int kRoom = (kSmemMaxPerCta - 8 * 1024 - NT * kQBytes) / kStage;
    static constexpr int kStages = kRoom > kMaxStages ? kMaxStages : kRoom;
    static constexpr int kSmem = 1024 + NT * kQBytes + kStages * kStage;
    // columns of tensor memory: S (two buffers, P in the same columns), then O
    static constexpr int kS = BN, kO = 2 * BN, kOStride = DB * 64;
    static_assert(kStages >= 3 && 2 * BN + NT * DB * 64 <= kTmemColsPerSm, "shape");
};

template <bool F16, int DB, int NT, int BN>
__global__ void __launch_bounds__(kThreads, 1)
attend_tile_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v)
{
    using Sh = TileShape<DB, NT, BN>;
    constexpr int ST = Sh::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 8];
    __shared__ uint16_t list[kMaxTiles];
    __shared__ __align__(16) int key_at[NT][2][BN];
    __shared__ int range_lo[2], range_hi[2], n_list, dead;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, kv_at = base + NT * Sh::kQBytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int i) { return bar0 + 8u * i; };
    const auto empty = [&](int i) { return bar0 + 8u * (kMaxStages + i); };
    const uint32_t q_full = bar0 + 8u * (2 * kMaxStages), s_full = q_full + 8, p_full = q_full + 24, o_full = q_full + 40;      // two of each
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;

    if (t == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
        mbar_init(q_full, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(p_full + 8 * i, 128); mbar_init(o_full + 8 * i, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < 2; ++i) { range_lo[i] = 0x7FFFFFFF; range_hi[i] = -1; }
        dead = 0;
    }
    if (warp == 9 && elect_one()) { prefetch_tensormap(&map_q); prefetch_tensormap(&map_k); prefetch_tensormap(&map_v); }
    pdl_wait();
    // (only now: what holds tensor memory ahead of this kernel in the stream is complete, and nothing that holds some waits for this CTA)
    if (warp == 9) tmem_alloc(smem_u32(&tmem_base), kTmemColsPerSm);
    // the block: the last ones, which see most keys, first
    const int heads = a.n_heads / a.pack, blk = a.n_blocks - 1 - static_cast<int>(blockIdx.x) / heads, head0 = static_cast<int>(blockIdx.x) % heads * a.pack;
    const AttSeq& s = a.s[seq_of_block(a, blk)];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack;      // queries of a tile
    const int q0 = (blk - s.blk0) * NT * per, len = seq_len(a, s);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    // this thread's row (softmax warps)
    const int tile = warp / 4, r = t & 127, i_row = q0 + tile * per + r / a.pack, head = head0 + r % a.pack;
    const bool mine = warp < 4 * NT && r < per * a.pack && i_row < s.n_q;
    const int p = mine ? query_pos(a, s, len, i_row) : -1;
    if (warp < 4 * NT) {
        const int lo = __reduce_min_sync(0xffffffffu, mine ? p : 0x7FFFFFFF), hi = __reduce_max_sync(0xffffffffu, p);
        if (lane == 0) { atomicMin(&range_lo[tile], lo); atomicMax(&range_hi[tile], hi); }
    }
    __syncthreads();
    const int lo0 = range_lo[0], hi0 = range_hi[0], lo1 = NT > 1 ? range_lo[1] : 0x7FFFFFFF, hi1 = NT > 1 ? range_hi[1] : -1;
    const TileRange range = tile_range(a, len, min(lo0, lo1), max(hi0, hi1), BN);
    const int per_split = (range.count + a.splits - 1) / a.splits, v0 = static_cast<int>(blockIdx.y) * per_split;
    const int n_range = max(0, min(range.count - v0, per_split));
    if (a.kv_pos) {
        for (int v = warp; v < n_range; v += kThreads / 32) {
            const Span k = key_span(a, s, len, range.tile(v0 + v) * BN, BN, lane);
            const int f = span_flags(a, lo0, hi0, k) | (NT > 1 ? span_flags(a, lo1, hi1, k) << 1 : 0);
            if (lane == 0) list[v] = static_cast<uint16_t>(f | (k.hidden ? kHidden : 0));
        }
    } else {
        for (int v = t; v < n_range; v += kThreads) {
            const Span k = counted_span(len, range.tile(v0 + v) * BN, BN);
            list[v] = static_cast<uint16_t>(span_flags(a, lo0, hi0, k) | (NT > 1 ? span_flags(a, lo1, hi1, k) << 1 : 0) | (k.hidden ? kHidden : 0));
        }
    }
    __syncthreads();
    if (warp == 0) {
        const int n = compact_entries(list, n_range, lane);
        if (lane == 0) n_list = n;
    }
    __syncthreads();
    const int n = n_list;
    const uint32_t tmem = tmem_base;
    Guard guard = {&dead, a.status};

    if (warp == 8) {
        if (n > 0 && elect_one()) {
            const int tiles = NT > 1 && q0 + per < s.n_q ? 2 : 1;
            mbar_expect_tx(q_full, tiles * DB * per * a.pack * 128);
            for (int i = 0; i < tiles; ++i)
                for (int b = 0; b < DB; ++b) tma_load_3d(q_at + i * Sh::kQBytes + b * kRows * 128, &map_q, b * 64, head0, s.qm_row + q0 + i * per, q_full);
            int c = 0;                                       // tiles of keys and values in turn
            for (; c < 2 * n; ++c) {
                const int st = c % ST;
                if (c >= ST && !guard.wait(empty(st), (c / ST - 1) & 1)) break;
                const int row = s.km_row + range.tile(v0 + (list[c / 2] >> kEntryShift)) * BN;
                mbar_expect_tx(full(st), Sh::kStage);
                for (int b = 0; b < DB; ++b) tma_load_3d(kv_at + st * Sh::kStage + b * BN * 128, c & 1 ? &map_v : &map_k, b * 64, hk, row, full(st));
            }
            if (c < 2 * n) {                                 // given up: what is under way has to land before the CTA may end
                mbar_wait(q_full, 0);
                for (int i = max(0, c - ST); i < c; ++i) mbar_wait(full(i % ST), i / ST & 1);
            }
        }
    } else if (warp == 9 && n > 0) {
        const uint32_t idesc_s = idesc_16<F16>(BN), idesc_o = idesc_16<F16>(a.head_dim) | kRowsAreContraction;
        const int steps = a.head_dim / 16;                   // of the contraction over the head
        const auto scores = [&](int i, int tl, int buf) {    // S of list entry i
            const int st = 2 * i % ST;
            for (int b = 0; b < DB; ++b)
                umma_box(2, tmem + buf * Sh::kS, smem_desc_sw128(q_at + tl * Sh::kQBytes + b * kRows * 128), smem_desc_sw128(kv_at + st * Sh::kStage + b * BN * 128),
                         idesc_s, min(4, steps - 4 * b), b > 0);
            umma_commit(s_full + 8 * buf);
        };
        const auto values = [&](int i, int tl, int buf, bool more) {
            const int st = (2 * i + 1) % ST;
            for (int k = 0; k < BN / 16; ++k)
                umma_bf16_ts(tmem + Sh::kO + tl * Sh::kOStride, tmem + buf * Sh::kS + 8 * k, smem_desc_rows_sw128(kv_at + st * Sh::kStage + k * 2048, BN * 128), idesc_o, more || k > 0);
        };
        const bool one = elect_one();
        int done[2] = {0, 0};                                // tiles whose P was taken, by tile of rows (NT = 2) or S buffer (NT = 1)
        bool any[2] = {false, false};
        bool ok = guard.wait_all(q_full, 0) && guard.wait_all(full(0), 0);
        if (ok && one) {
            tc_fence_after();
            for (int tl = 0; tl < NT; ++tl)
                if (list[0] >> tl & kNeed) scores(0, tl, tl);
            umma_commit(empty(0));
        }
        for (int i = 0; i < n && ok; ++i) {
            const int e = list[i], next = i + 1 < n ? list[i + 1] : 0;
            if (NT == 1 && i + 1 < n) {
                ok = guard.wait_all(full((2 * i + 2) % ST), (2 * i + 2) / ST & 1);
                if (!ok) break;
                if (one) {
                    tc_fence_after();
                    scores(i + 1, 0, (i + 1) & 1);
                    umma_commit(empty((2 * i + 2) % ST));
                }
            }
            const int st = (2 * i + 1) % ST;
            ok = guard.wait_all(full(st), (2 * i + 1) / ST & 1);
            if (!ok) break;
            if (e & kHidden) {                               // values that nobody may look at become zero
                const int j0 = range.tile(v0 + (e >> kEntryShift)) * BN;
                for (int k = lane; k < BN; k += 32) {
                    if (key_pos(a, s, len, j0 + k) >= 0) continue;
                    for (int b = 0; b < DB; ++b)
                        for (int c = 0; c < 8; ++c)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(kv_at + st * Sh::kStage + b * BN * 128 + k * 128 + c * 16), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            if (NT == 2 && i + 1 < n) {
                ok = guard.wait_all(full((2 * i + 2) % ST), (2 * i + 2) / ST & 1);
                if (!ok) break;
            }
            for (int tl = 0; tl < NT && ok; ++tl) {
                const int buf = NT == 2 ? tl : i & 1;
                if (e >> tl & kNeed) {
                    ok = guard.wait_all(p_full + 8 * buf, done[buf]++ & 1);
                    if (!ok) break;
                    if (one) {
                        tc_fence_after();
                        values(i, tl, buf, any[tl]);
                        if (NT == 1) umma_commit(o_full);    // (every step: the softmax warps look at it when they move the reference)
                    }
                    any[tl] = true;
                }
                if (NT == 2 && one && (next >> tl & kNeed)) scores(i + 1, tl, tl);
            }
            if (ok && one) {
                umma_commit(empty(st));
                if (NT == 2 && i + 1 < n) umma_commit(empty((2 * i + 2) % ST));
            }
            __syncwarp();
        }
        if (ok && one) {                                     // everything is in O (NT = 1: on the second barrier, the first one counts steps)
            if (NT == 2) umma_commit(o_full);
            umma_commit(o_full + 8);
        }
        __syncwarp();
    } else if (warp < 4 * NT) {
        // ---- softmax of a tile of rows, a thread per row
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;        // this warp's 32 lanes
        const uint32_t o_col = tmem + Sh::kO + tile * Sh::kOStride + lanes;
        const float scale = a.scale_log2;
        float m = -CUDART_INF_F, l = 0.f;                    // reference (scaled), sum
        int seen = 0;                                        // tiles so far
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int e = list[i];
            if (!(e >> tile & kNeed)) continue;
            const int buf = NT == 2 ? tile : seen & 1, turn = NT == 2 ? seen : seen >> 1;
            uint32_t visible[BN / 32];                       // a bit for every key of the tile that the row sees
            if (e >> tile & kMask) {
                const int j0 = range.tile(v0 + (e >> kEntryShift)) * BN;
                if (a.kv_pos) {                              // the positions for the four warps (two buffers: one barrier a tile is enough)
                    int* const at = key_at[tile][seen & 1];
                    if (r < BN) at[r] = key_pos(a, s, len, j0 + r);
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + tile) : "memory");
#pragma unroll
                    for (int w = 0; w < BN / 32; ++w) {
                        uint32_t bits = 0;
#pragma unroll 8
                        for (int c = 0; c < 32; ++c) bits |= sees(p, at[32 * w + c], a.window, a.n_sink) ? 1u << c : 0u;
                        visible[w] = bits;
                    }
                } else {
                    const int past = min(p, len - 1) - j0 + 1, first = max(p - a.window + 1, 0) - j0, sink = a.n_sink - j0;
#pragma unroll
                    for (int w = 0; w < BN / 32; ++w) visible[w] = below(past - 32 * w) & (~below(first - 32 * w) | below(sink - 32 * w));
                }
            }
            ok = guard.wait_all(s_full + 8 * buf, turn & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t s_col = tmem + buf * Sh::kS + lanes;
            float x[BN];
            tmem_ld_cols<BN>(s_col, x);
            if (e >> tile & kMask) {
#pragma unroll
                for (int c = 0; c < BN; ++c) x[c] = visible[c / 32] >> (c & 31) & 1u ? x[c] : -CUDART_INF_F;
            }
            float tops[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int c = 4; c < BN; ++c) tops[c & 3] = fmaxf(tops[c & 3], x[c]);
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * scale;      // (scale is positive)
            const bool move = top > m + kMoveAt;
            if (seen > 0 && __any_sync(0xffffffffu, move)) {
                // (one tile of rows: the step before may still be adding; the one before that was complete before this S was)
                if (NT == 1) ok = guard.wait_all(o_full, (seen - 1) & 1);
                if (!ok) break;
                tc_fence_after();
                const float f = move ? ex2_approx(m - top) : 1.f;
#pragma unroll 1
                for (int c = 0; c < a.head_dim; c += 16) {
                    float o[16];
                    uint32_t w[16];
                    tmem_ld_cols<16>(o_col + c, o);
#pragma unroll
                    for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * f);
                    tmem_st_cols<16>(o_col + c, w);
                }
                l *= f;
            }
            if (move) m = top;
            const float ref = m == -CUDART_INF_F ? 0.f : m;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c0 = 0; c0 < BN; c0 += 32) {
                uint32_t w[16];
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float y = ex2_approx(fmaf(x[c0 + c], scale, -ref)), z = ex2_approx(fmaf(x[c0 + c + 1], scale, -ref));
                    sum[c & 2] += y;
                    sum[(c & 2) + 1] += z;
                    w[c / 2] = F16 ? two_f16(y, z) : two_bf16(y, z);
                }
                tmem_st_cols<16>(s_col + c0 / 2, w);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(p_full + 8 * buf);
            ++seen;
        }
        // ---- the tile's rows
        if (ok && seen > 0) ok = guard.wait_all(o_full + 8 * (NT == 2 ? tile : 1), 0);
        tc_fence_after();
        const int64_t part = s.part0 + static_cast<int64_t>(blockIdx.y) * s.n_q + i_row;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        for (int c = 0; c < a.head_dim && ok; c += 32) {
            float o[32];
            if (seen > 0) tmem_ld_cols<32>(o_col + c, o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = l > 0.f ? (a.splits > 1 ? o[k] : o[k] * inv) : 0.f;
            if (!mine) continue;
            if (a.splits > 1) {
                float* const dst = a.part_o + (part * a.n_heads + head) * a.head_dim + c;
#pragma unroll
                for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            } else {
                __nv_bfloat16* const dst = static_cast<__nv_bfloat16*>(a.out) + ((s.q_row + i_row) * a.n_heads + head) * a.head_dim + c;
#pragma unroll
                for (int k = 0; k < 32; k += 8) store8(dst + k, o + k);
            }
        }
        if (mine && ok) {
            if (a.splits > 1) {
                a.part_ml[part * a.n_heads + head] = make_float2(m, l);
            } else {
                const float z = l > 0.f ? m + log2f(l) : -CUDART_INF_F;
                if (a.lse) a.lse[(s.q_row + i_row) * a.n_heads + head] = z * 0.69314718055994531f;      // ln 2
                if (a.mass) a.lse2[static_cast<int64_t>(s.qp0 + i_row) * a.n_heads + head] = z;
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemColsPerSm);
    }
}

// attend_weights_kernel: mass of 128 cached rows over the queries of their sequence, for the heads packed together.  Keys on the lanes
// of tensor memory, queries on its columns: S^T = K Q^T, and a thread adds up 2^(S - lse) over the columns of its key, so that
// no sum crosses threads.  Tiles of queries go to the two groups of four warps in turn; four buffers of S.
constexpr int kQStages = 4;

template <int DB>
struct WeightShape {
    static constexpr int kTileBytes = DB * kRows * 128;
    static constexpr int kRoom = (kSmemMaxPerCta - 16 * 1024 - kTileBytes) / kTileBytes;
    static constexpr int kStages = kRoom > kQStages ? kQStages : kRoom;
    // (at least what keeps a second CTA, which would find no tensor memory, off the multiprocessor)
    static constexpr int kUsed = 1024 + (1 + kStages) * kTileBytes;
    static constexpr int kSmem = kUsed > 120 * 1024 ? kUsed : 120 * 1024;
    static_assert(kStages >= 2, "shape");
};

template <bool F16, int DB>
__global__ void __launch_bounds__(kThreads, 1)
attend_weights_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap)
{
    using Sh = WeightShape<DB>;
    constexpr int ST = Sh::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kQStages + 9];
    __shared__ uint16_t list[kMaxTiles];
    __shared__ __align__(16) float row_z[4][kRows];
    __shared__ int row_p[4][kRows];
    __shared__ float half[kRows];
    __shared__ int n_list, dead;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t k_at = base, q_at = base + Sh::kTileBytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int i) { return bar0 + 8u * i; };
    const auto empty = [&](int i) { return bar0 + 8u * (kQStages + i); };
    const uint32_t s_full = bar0 + 8u * (2 * kQStages), s_empty = s_full + 32, k_full = s_full + 64;      // four of each S buffer's
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    if (t == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
        for (int i = 0; i < 4; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(s_empty + 8 * i, 128); }
        mbar_init(k_full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead = 0;
    }
    if (warp == 9 && elect_one()) { prefetch_tensormap(&map_q); prefetch_tensormap(&map_k); }
    pdl_wait();
    if (warp == 9) tmem_alloc(smem_u32(&tmem_base), kTmemColsPerSm);
    const int packs = a.n_heads / a.pack, pk = static_cast<int>(blockIdx.x) % packs, head0 = pk * a.pack;
    int b = 0, tile = static_cast<int>(blockIdx.x) / packs;
    while (b + 1 < a.n_seq && tile >= (a.s[b].n_kv + kRows - 1) / kRows) tile -= (a.s[b++].n_kv + kRows - 1) / kRows;
    const AttSeq& s = a.s[b];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack, len = seq_len(a, s), j0 = tile * kRows;
    const int q_tiles = (s.n_q + per - 1) / per, v0 = static_cast<int>(blockIdx.y) * kMaxTiles, n_range = max(0, min(q_tiles - v0, kMaxTiles));
    // the tiles of queries some of which see some of these keys
    const Span k = a.kv_pos ? key_span(a, s, len, j0, kRows, lane) : counted_span(len, j0, kRows);
    const auto tile_flags = [&](int v, int lo, int hi) {
        const bool whole = (v + 1) * per <= s.n_q && per * a.pack == kRows;
        const int f = span_flags(a, lo, hi, k);
        return f && !whole ? f | kMask : f;
    };
    if (a.q_pos) {
        for (int v = warp; v < n_range; v += kThreads / 32) {
            int lo = 0x7FFFFFFF, hi = -1;
            for (int i = (v0 + v) * per + lane; i < min((v0 + v + 1) * per, s.n_q); i += 32) {
                const int p = query_pos(a, s, len, i);
                lo = min(lo, p);
                hi = max(hi, p);
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (lane == 0) list[v] = static_cast<uint16_t>(tile_flags(v0 + v, lo, hi));
        }
    } else {
        for (int v = t; v < n_range; v += kThreads)
            list[v] = static_cast<uint16_t>(tile_flags(v0 + v, query_pos(a, s, len, (v0 + v) * per), query_pos(a, s, len, min((v0 + v + 1) * per, s.n_q) - 1)));
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    if (warp == 0) {
        const int c = compact_entries(list, n_range, lane);
        if (lane == 0) n_list = c;
    }
    __syncthreads();
    const int n = n_list;
    const uint32_t tmem = tmem_base;
    Guard guard = {&dead, a.status};
    const int row_bytes = per * a.pack * 128;

    if (warp == 8) {
        if (n > 0 && elect_one()) {
            mbar_expect_tx(k_full, Sh::kTileBytes);
            for (int i = 0; i < DB; ++i) tma_load_3d(k_at + i * kRows * 128, &map_k, i * 64, hk, s.km_row + j0, k_full);
            int c = 0;
            for (; c < n; ++c) {
                const int st = c % ST;
                if (c >= ST && !guard.wait(empty(st), (c / ST - 1) & 1)) break;
                mbar_expect_tx(full(st), DB * row_bytes);
                for (int i = 0; i < DB; ++i) tma_load_3d(q_at + st * Sh::kTileBytes + i * kRows * 128, &map_q, i * 64, head0, s.qm_row + (v0 + (list[c] >> kEntryShift)) * per, full(st));
            }
            if (c < n) {
                mbar_wait(k_full, 0);
                for (int i = max(0, c - ST); i < c; ++i) mbar_wait(full(i % ST), i / ST & 1);
            }
        }
    } else if (warp == 9) {
        const uint32_t idesc = idesc_16<F16>(kRows);
        const int steps = a.head_dim / 16;
        const bool one = elect_one();
        bool ok = n == 0 || guard.wait_all(k_full, 0);
        for (int i = 0; i < n && ok; ++i) {
            const int st = i % ST, buf = i & 3;
            ok = guard.wait_all(full(st), i / ST & 1) && (i < 4 || guard.wait_all(s_empty + 8 * buf, (i / 4 - 1) & 1));
            if (ok && one) {
                tc_fence_after();
                for (int c = 0; c < DB; ++c)
                    umma_box(2, tmem + buf * kRows, smem_desc_sw128(k_at + c * kRows * 128), smem_desc_sw128(q_at + st * Sh::kTileBytes + c * kRows * 128), idesc,
                             min(4, steps - 4 * c), c > 0);
                umma_commit(s_full + 8 * buf);
                umma_commit(empty(st));
            }
            __syncwarp();
        }
    } else {
        const int group = warp / 4, r = t & 127, j = j0 + r;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;
        const int c_pos = key_pos(a, s, len, j);
        const float scale = a.scale_log2;
        float sum = 0.f;
        bool ok = true;
        for (int i = group; i < n && ok; i += 2) {
            const int buf = i & 3, e = list[i];
            {                                                // this thread's query row: for all keys of the group
                const int iq = (v0 + (e >> kEntryShift)) * per + r / a.pack;
                const bool there = r < per * a.pack && iq < s.n_q;
                row_p[buf][r] = there ? query_pos(a, s, len, iq) : -1;
                row_z[buf][r] = there ? a.lse2[static_cast<int64_t>(s.qp0 + iq) * a.n_heads + head0 + r % a.pack] : 0.f;
            }
            asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
            ok = guard.wait_all(s_full + 8 * buf, i / 4 & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t s_col = tmem + buf * kRows + lanes;
            float part[4] = {0.f, 0.f, 0.f, 0.f};
            const bool masked = (e & kMask) != 0;
#pragma unroll
            for (int c0 = 0; c0 < kRows; c0 += 32) {
                float x[32];
                tmem_ld_cols<32>(s_col + c0, x);
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const float y = ex2_approx(fmaf(x[c], scale, -row_z[buf][c0 + c]));
                        part[c & 3] += sees(row_p[buf][c0 + c], c_pos, a.window, a.n_sink) ? y : 0.f;
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float4 z = *reinterpret_cast<const float4*>(&row_z[buf][c0 + c]);
                        part[0] += ex2_approx(fmaf(x[c], scale, -z.x));
                        part[1] += ex2_approx(fmaf(x[c + 1], scale, -z.y));
                        part[2] += ex2_approx(fmaf(x[c + 2], scale, -z.z));
                        part[3] += ex2_approx(fmaf(x[c + 3], scale, -z.w));
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(s_empty + 8 * buf);
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        if (group == 1) half[r] = sum;
        asm volatile("bar.sync 3, 256;" ::: "memory");
        if (group == 0 && j < s.n_kv)
            a.part_mass[(static_cast<int64_t>(blockIdx.y) * packs + pk) * a.total_kv + s.kvp0 + j] = sum + half[r];
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemColsPerSm);
    }
}

template <class K>
cudaError_t launch(KernelSetup& setup, K kernel, dim3 grid, size_t smem, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(kernel), smem, kTmemColsPerSm);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, maps.q, maps.k, maps.v);
}

template <bool F16, int DB, int NT, int BN>
cudaError_t attend(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    static KernelSetup setup;
    const dim3 grid(static_cast<unsigned>(a.n_blocks) * static_cast<unsigned>(a.n_heads / a.pack), static_cast<unsigned>(a.splits));
    return launch(setup, attend_tile_kernel<F16, DB, NT, BN>, grid, TileShape<DB, NT, BN>::kSmem, a, maps, stream);
}

template <bool F16, int DB>
cudaError_t weights(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    static KernelSetup setup;
    int64_t tiles = 0;
    for (int b = 0; b < a.n_seq; ++b) tiles += (a.s[b].n_kv + kRows - 1) / kRows;
    if (tiles == 0) return cudaSuccess;
    const int packs = a.n_heads / a.pack;
    return launch(setup, attend_weights_kernel<F16, DB>, dim3(static_cast<unsigned>(tiles * packs), static_cast<unsigned>(a.mass_parts / packs)), WeightShape<DB>::kSmem, a, maps, stream);
}

// e4m3 rows of the sequences as fp16 rows, packed (exact).  A thread converts 16 elements at a time.
__global__ void __launch_bounds__(256) widen_kernel(const __grid_constant__ AttArgs a, uint8_t* wide_q, uint8_t* wide_k, uint8_t* wide_v)
{
    pdl_wait();
    pdl_trigger();
    const int qw = a.n_heads * a.head_dim / 16, kw = a.kv_heads * a.head_dim / 16;
    const int64_t nq = static_cast<int64_t>(a.total_q) * qw, nk = static_cast<int64_t>(a.total_kv) * kw;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; u < nq + 2 * nk; u += stride) {
        const int what = u < nq ? 0 : u < nq + nk ? 1 : 2;
        const int64_t v = what == 0 ? u : what == 1 ? u - nq : u - nq - nk;
        const int w = what == 0 ? qw : kw;
        const int row = static_cast<int>(v / w), c = static_cast<int>(v - static_cast<int64_t>(row) * w);
        int b = 0;
        while (b + 1 < a.n_seq && row >= (what == 0 ? a.s[b + 1].qp0 : a.s[b + 1].kvp0)) ++b;
        const int64_t src_row = what == 0 ? a.s[b].q_row + row - a.s[b].qp0 : a.s[b].kv_row + row - a.s[b].kvp0;
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(what == 0 ? a.q : what == 1 ? a.k : a.v) + (src_row * w + c) * 16);
        const uint32_t in[4] = {x.x, x.y, x.z, x.w};
        uint32_t out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(in[i / 2] >> (16 * (i & 1))), __NV_E4M3);
            out[i] = static_cast<uint32_t>(h.x) | static_cast<uint32_t>(h.y) << 16;
        }
        uint4* const dst = reinterpret_cast<uint4*>((what == 0 ? wide_q : what == 1 ? wide_k : wide_v) + (static_cast<int64_t>(row) * w + c) * 32);
        dst[0] = make_uint4(out[0], out[1], out[2], out[3]);
        dst[1] = make_uint4(out[4], out[5], out[6], out[7]);
    }
}

}  // namespace

cudaError_t launch_widen(const AttArgs& a, void* wide_q, void* wide_k, void* wide_v, cudaStream_t stream)
{
    const int64_t units = (static_cast<int64_t>(a.total_q) * a.n_heads + 2 * static_cast<int64_t>(a.total_kv) * a.kv_heads) * a.head_dim / 16;
    if (units == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>((units + 255) / 256, 16 * sm_count_of_current_device())));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, widen_kernel, a, static_cast<uint8_t*>(wide_q), static_cast<uint8_t*>(wide_k), static_cast<uint8_t*>(wide_v));
}

namespace {
template <bool F16>
cudaError_t weights_by_dim(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    switch ((a.head_dim + 63) / 64) {
    case 1: return weights<F16, 1>(a, maps, stream);
    case 2: return weights<F16, 2>(a, maps, stream);
    case 3: return weights<F16, 3>(a, maps, stream);
    default: return weights<F16, 4>(a, maps, stream);
    }
}
template <bool F16>
cudaError_t attend_by_dim(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    switch ((a.head_dim + 63) / 64) {
    case 1: return attend<F16, 1, 2, 128>(a, maps, stream);
    case 2: return attend<F16, 2, 2, 128>(a, maps, stream);
    case 3: return attend<F16, 3, 1, 64>(a, maps, stream);
    default: return attend<F16, 4, 1, 64>(a, maps, stream);
    }
}
}  // namespace

cudaError_t launch_attend_weights(bool f16, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    return f16 ? weights_by_dim<true>(a, maps, stream) : weights_by_dim<false>(a, maps, stream);
}

cudaError_t launch_attend_tile(bool f16, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    return f16 ? attend_by_dim<true>(a, maps, stream) : attend_by_dim<false>(a, maps, stream);
}

}  // namespace mvla
