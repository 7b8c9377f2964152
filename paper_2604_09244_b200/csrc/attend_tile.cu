// Windowed attention of blocks of queries on the tensor cores (bf16; e4m3 widened to fp16), and the weights that it gives to the cached rows.
//
// attend_tile_kernel.  A CTA has a tile of 128 query rows that share a key head (row r: query r / g, head r % g of the g heads
// packed side by side, one TMA box) and walks the tiles of 64 keys that some of its rows may see:
//     S = Q K^T (tcgen05, both from shared memory)  ->  P = 2^(S - reference), rounded to 16 bits, back into the columns of S
//     ->  O += P V (tcgen05, P from tensor memory, V as it lies in the cache: its rows are the contraction).
// fp16 weights (e4m3 rows) are counted in units of 2^-kF16Lift of the reference, so that faint ones stay normal numbers as long as can be.
// Warps 0-3: the softmax, a thread per row: maximum and sum without a shuffle.  The sums in O are taken against a reference that is
// moved only when a row's maximum grows past it by 2^8 (the result is the same; moving it is a pass over O).  Warp 4 loads, warp 5
// issues the MMAs; S is double-buffered, so that the next scores are there when the softmax of the last ones ends.
// Heads of up to 128 elements leave room for two CTAs to a multiprocessor (256 columns of tensor memory, 97 KB of shared memory each):
// one's exponentials, prologue and epilogue lie beside the other's MMAs.  Measured on 8192 queries, 16 heads of 128 in groups of 4, and on
// 16 x 808 queries of 32 heads, window 512: two tiles of rows in one CTA with tiles of 128 keys 295 / 250 us, this 291 / 189.
// Now 305 us (900 TFLOP/s; copies of the kernel without all but the MMAs 235, without the exponentials 286: reads of shared memory by 64-key MMAs, and
// the chain from scores to weights; the tensor cores are busy half of the time, and so are the pipes of the exponentials) and 195 + 135 for the weights.  Single tokens without weights come here too: 131072 rows of 8 heads of 128 99.9 us, 5.4 TB/s.
// Positions that are counted tell every warp which tiles to visit and which need their mask; where they are data, a list of the
// tiles is made first.  Keys that no row of the tile sees have their values set to zero in shared memory (0 times NaN is NaN).
#include "attend.cuh"
#include "attend_walk.h"
#include "f32x2.cuh"
#include "tmem_ld.cuh"
#include "tmem_plan.h"
#include "tmem_st.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 320;                // attend_weights_kernel
constexpr int kRows = 128;                   // query rows of a tile
constexpr int kKeys = 64;                    // keys of a tile
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

// What a tile of keys (or queries) is to a CTA: some row sees some key, not every row sees every key.
constexpr int kNeed = 1, kMask = 2, kEntryShift = 2;         // an entry of a list: the tile's place in the range above the flags
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
        const unsigned on = __ballot_sync(0xffffffffu, (f & kNeed) != 0);
        __syncwarp();
        if (f & kNeed) list[count + __popc(on & ((1u << lane) - 1u))] = static_cast<uint16_t>((i0 + lane) << kEntryShift | f);
        __syncwarp();
        count += __popc(on);
    }
    return count;
}

// Bounded waits of a CTA: when one runs out, the others end without waiting for long, and warps that meet one another go on meeting
// (attend_walk.h).  Before the CTA ends, the loads and the MMAs that are under way do: also with a limit.
struct Guard {
    int* dead;
    int* status;
    // by a whole warp: the same answer in all its lanes
    __device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)); }
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity)
    {
        if (mbar_try_wait<false>(bar, parity)) return true;
        return !*reinterpret_cast<volatile int*>(dead) && spin(bar, parity);
    }
    // of what is under way, whoever gave up
    __device__ __forceinline__ void settle(uint32_t bar, uint32_t parity)
    {
        if (!mbar_try_wait<false>(bar, parity)) spin(bar, parity);
    }
    __device__ __forceinline__ bool spin(uint32_t bar, uint32_t parity)
    {
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

// Smallest and largest position of queries [i0, i1) of a sequence, by one warp.
__device__ __forceinline__ void query_span(const AttArgs& a, const AttSeq& s, int len, int i0, int i1, int lane, int* lo, int* hi)
{
    if (!a.q_pos) {
        *lo = query_pos(a, s, len, i0);
        *hi = query_pos(a, s, len, i1 - 1);
        return;
    }
    int l = 0x7FFFFFFF, h = -1;
    for (int i = i0 + lane; i < i1; i += 32) {
        const int p = query_pos(a, s, len, i);
        l = min(l, p);
        h = max(h, p);
    }
    *lo = __reduce_min_sync(0xffffffffu, l);
    *hi = __reduce_max_sync(0xffffffffu, h);
}

template <int DB>
struct TileShape {
    static constexpr int kWarps = 6, kLoads = 4, kIssues = 5;
    // columns of tensor memory: S (two buffers, P in the same columns), then O
    static constexpr int kO = 2 * kKeys, kColumns = kO + DB * 64 <= 256 ? 256 : 512;
    static constexpr int kCtas = kTmemColsPerSm / kColumns;  // to a multiprocessor
    static constexpr int kQBytes = DB * kRows * 128;
    static constexpr int kStage = DB * kKeys * 128;          // one tile of keys or values
    static constexpr int kRoom = ((kCtas == 2 ? kSmemPerSm / 2 - kSmemReservedPerCta : kSmemMaxPerCta) - 8 * 1024 - kQBytes) / kStage;
    static constexpr int kStages = kRoom > kMaxStages ? kMaxStages : kRoom;
    static constexpr int kSmem = 1024 + kQBytes + kStages * kStage;
    static_assert(kStages >= 4, "shape");
};

// TOKENS: bf16 weights of sequences that count as single tokens meet the values in two parts, what the type holds and what it leaves.  Such a sequence
// has kTokenRows of the tile's 128 rows at most, so its query rows are there twice, kTwin rows apart: the first ones' row of P takes the one part, their
// twin's the other, and the rows of O are added up at the end.  No MMA more, and none of the other rows' exponentials.
constexpr int kTwin = 32;                    // (a warp's lanes)
static_assert(kTokenRows <= kTwin, "the rows of a warp");

template <bool F16, int DB, bool TOKENS>
__global__ void __launch_bounds__(TileShape<DB>::kWarps * 32, TileShape<DB>::kCtas)
attend_tile_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v)
{
    using Sh = TileShape<DB>;
    constexpr int ST = Sh::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 8];
    __shared__ uint16_t list[kMaxTiles];
    __shared__ int key_at[kKeys];
    __shared__ uint32_t seen_by[4][4][kKeys / 32];           // of the last tiles: the keys that some row of a warp sees
    __shared__ int n_list, dead;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, kv_at = base + Sh::kQBytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int i) { return bar0 + 8u * i; };
    const auto empty = [&](int i) { return bar0 + 8u * (kMaxStages + i); };
    // s_full, p_full: of each S buffer; o_step: a step's values are in O; o_full: all are; ended: the MMAs of a CTA that gave up
    const uint32_t q_full = bar0 + 8u * (2 * kMaxStages), s_full = q_full + 8, p_full = q_full + 24, o_step = q_full + 40, o_full = q_full + 48,
                   ended = q_full + 56;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;

    if (warp == Sh::kLoads && lane == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
        mbar_init(q_full, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(p_full + 8 * i, 128); }
        mbar_init(o_step, 1);
        mbar_init(o_full, 1);
        mbar_init(ended, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        dead = 0;
        prefetch_tensormap(&map_q);
        if (a.total_kv > 0) {                                // (else these two are no tensor maps)
            prefetch_tensormap(&map_k);
            prefetch_tensormap(&map_v);
        }
    }
    __syncwarp();
    pdl_wait();
    // (only now: what holds tensor memory ahead of this kernel in the stream is complete, and nothing that holds some waits for this CTA)
    if (warp == Sh::kIssues) tmem_alloc(smem_u32(&tmem_base), Sh::kColumns);
    // the block: the last ones, which see most keys, first
    const int heads = a.n_heads / a.pack, blk = a.n_blocks - 1 - static_cast<int>(blockIdx.x) / heads, head0 = static_cast<int>(blockIdx.x) % heads * a.pack;
    const AttSeq& s = a.s[seq_of_block(a, blk)];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack;      // queries of the tile
    const int q0 = (blk - s.blk0) * per, len = seq_len(a, s);
    const bool twins = TOKENS && static_cast<int64_t>(s.n_q) * (a.n_heads / a.kv_heads) <= kTokenRows;
    int lo, hi;
    query_span(a, s, len, q0, min(q0 + per, s.n_q), lane, &lo, &hi);
    const TileRange range = tile_range(a, len, lo, hi, kKeys);
    const int per_split = (range.count + a.splits - 1) / a.splits, v0 = static_cast<int>(blockIdx.y) * per_split;
    int n = max(0, min(range.count - v0, per_split));
    if (a.kv_pos) {
        for (int v = warp; v < n; v += Sh::kWarps) {
            const Span k = key_span(a, s, len, range.tile(v0 + v) * kKeys, kKeys, lane);
            if (lane == 0) list[v] = static_cast<uint16_t>(span_flags(a, lo, hi, k));
        }
        __syncthreads();
        if (warp == 0) {
            const int c = compact_entries(list, n, lane);
            if (lane == 0) n_list = c;
        }
        __syncthreads();
        n = n_list;
    }
    // the i-th tile: where its keys begin, and what it is (counted positions: all tiles of the range are visited)
    const auto first_key = [&](int i) { return range.tile(v0 + (a.kv_pos ? list[i] >> kEntryShift : i)) * kKeys; };
    const auto flags_of = [&](int i, int j0) {
        if (a.kv_pos) return static_cast<int>(list[i]);
        const Span k = counted_span(len, j0, kKeys);
        const int f = span_flags(a, lo, hi, k);              // (queries far apart may leave out a tile between them: then no row sees a key)
        return f ? f : kMask;
    };
    Guard guard = {&dead, a.status};

    // ---- loads (one lane of a warp): the first ones before the CTA meets
    const auto load = [&](int c) {                           // tiles of keys and values in turn
        const int st = c % ST, row = s.km_row + first_key(c / 2);
        mbar_expect_tx(full(st), Sh::kStage);
        for (int b = 0; b < DB; ++b) tma_load_3d(kv_at + st * Sh::kStage + b * kKeys * 128, c & 1 ? &map_v : &map_k, b * 64, hk, row, full(st));
    };
    const int at_once = min(ST, 2 * n);
    if (warp == Sh::kLoads && lane == 0 && n > 0) {
        mbar_expect_tx(q_full, DB * per * a.pack * 128);
        for (int b = 0; b < DB; ++b) tma_load_3d(q_at + b * kRows * 128, &map_q, b * 64, head0, s.qm_row + q0, q_full);
        for (int c = 0; c < at_once; ++c) load(c);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base;

    if (warp == Sh::kLoads) {
        if (lane == 0 && n > 0) {
            int c = at_once;
            for (; c < 2 * n; ++c) {
                if (!guard.wait(empty(c % ST), (c / ST - 1) & 1)) break;
                load(c);
            }
            guard.settle(q_full, 0);                         // (whoever gave up, what is under way lands before the CTA ends)
            for (int i = max(0, c - ST); i < c; ++i) guard.settle(full(i % ST), i / ST & 1);
        }
    } else if (warp == Sh::kIssues && n > 0) {
        const uint32_t idesc_s = idesc_16<F16>(kKeys), idesc_o = idesc_16<F16>(a.head_dim) | kRowsAreContraction;
        const int steps = a.head_dim / 16;                   // of the contraction over the head
        const bool one = elect_one();
        const auto scores = [&](int i) {                     // S of tile i; its keys' stage is free when it is there
            const int st = 2 * i % ST;
            for (int b = 0; b < DB; ++b)
                umma_box(2, tmem + (i & 1) * kKeys, smem_desc_sw128(q_at + b * kRows * 128), smem_desc_sw128(kv_at + st * Sh::kStage + b * kKeys * 128), idesc_s,
                         min(4, steps - 4 * b), b > 0);
            umma_commit(s_full + 8 * (i & 1));
            umma_commit(empty(st));
        };
        bool ok = guard.wait_all(q_full, 0);
        if (TOKENS && twins && ok) {                         // (whole swizzled groups of eight rows: they lie alike kTwin rows on)
            constexpr int kPer = kTokenRows * 8 / 32;        // 16-byte pieces of a lane in a box
            uint32_t w[DB * kPer][4];
#pragma unroll
            for (int u = 0; u < DB * kPer; ++u)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[u][0]), "=r"(w[u][1]), "=r"(w[u][2]), "=r"(w[u][3])
                             : "r"(q_at + u / kPer * kRows * 128 + (u % kPer * 32 + lane) * 16) : "memory");
#pragma unroll
            for (int u = 0; u < DB * kPer; ++u)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_at + u / kPer * kRows * 128 + kTwin * 128 + (u % kPer * 32 + lane) * 16),
                             "r"(w[u][0]), "r"(w[u][1]), "r"(w[u][2]), "r"(w[u][3]) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        }
        ok = ok && guard.wait_all(full(0), 0);
        if (ok && one) {
            tc_fence_after();
            scores(0);
        }
        for (int i = 0; i < n && ok; ++i) {
            if (i + 1 < n) {
                ok = guard.wait_all(full((2 * i + 2) % ST), (2 * i + 2) / ST & 1);
                if (ok && one) {
                    tc_fence_after();
                    scores(i + 1);
                }
                __syncwarp();
            }
            const int c = 2 * i + 1, st = c % ST;
            ok = ok && guard.wait_all(full(st), c / ST & 1);
            if (!ok) break;
            const int j0 = first_key(i);
            if (flags_of(i, j0) & kMask) {
                // values that no row sees become zero: counted queries lie side by side, so that their span says it, others have to be asked
                uint32_t by[kKeys / 32] = {};
                if (a.q_pos) {
                    ok = guard.wait_all(p_full + 8 * (i & 1), i / 2 & 1);
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int x = 0; x < kKeys / 32; ++x) by[x] |= seen_by[i & 3][w][x];
                }
                bool some = false;
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x) {
                    const int k = 32 * x + lane;
                    if (a.q_pos ? by[x] >> lane & 1u : j0 + k < len && some_sees(lo, hi, j0 + k, a.window, a.n_sink)) continue;
                    some = true;
                    for (int c16 = 0; c16 < DB * 8; ++c16)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(kv_at + st * Sh::kStage + c16 / 8 * kKeys * 128 + k * 128 + c16 % 8 * 16), "r"(0) : "memory");
                }
                if (some) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            ok = ok && guard.wait_all(p_full + 8 * (i & 1), i / 2 & 1);
            if (ok && one) {
                tc_fence_after();
                for (int k = 0; k < kKeys / 16; ++k)
                    umma_bf16_ts(tmem + Sh::kO, tmem + (i & 1) * kKeys + 8 * k, smem_desc_rows_sw128(kv_at + st * Sh::kStage + k * 2048, kKeys * 128), idesc_o, i > 0 || k > 0);
                umma_commit(o_step);
                umma_commit(empty(st));
            }
            __syncwarp();
        }
        if (one) umma_commit(ok ? o_full : ended);
        __syncwarp();
        guard.settle(ok ? o_full : ended, 0);                   // (whoever else gave up, the tensor memory is not given back under an MMA)
    } else if (warp < 4) {
        // ---- softmax, a thread per row
        const int r = TOKENS && twins ? t % kTwin : t;       // row of the tile
        const bool twin = TOKENS && twins && t >= kTwin;     // (the rows from 2 kTwin on are nobody's)
        const int i_row = q0 + r / a.pack, head = head0 + r % a.pack;
        const bool mine = r < per * a.pack && i_row < s.n_q && !(TOKENS && twins && t >= 2 * kTwin);
        const int p = mine ? query_pos(a, s, len, i_row) : -1;
        const uint32_t lanes = static_cast<uint32_t>(warp) << 21;            // this warp's 32 lanes
        const uint32_t o_col = tmem + Sh::kO + lanes;
        const float scale = a.scale_log2;
        const uint64_t scale2 = two_f32(scale, scale);
        constexpr float kLift = F16 ? kF16Lift : 0.f;
        float m = -CUDART_INF_F, l = 0.f;                    // reference (scaled), sum (of weights against the reference less kLift)
        bool masked = false;
        uint32_t visible[kKeys / 32];                        // a bit for every key of the tile that the row sees
        const auto look = [&](int i) {
            const int j0 = first_key(i);
            masked = (flags_of(i, j0) & kMask) != 0;
            if (!masked) return;
            if (a.kv_pos) {                                  // the positions, for the four warps
                asm volatile("bar.sync 1, 128;" ::: "memory");       // (nobody reads the last ones any more)
                if (t < kKeys) key_at[t] = key_pos(a, s, len, j0 + t);
                asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
                for (int w = 0; w < kKeys / 32; ++w) {
                    uint32_t bits = 0;
#pragma unroll 8
                    for (int c = 0; c < 32; ++c) bits |= sees(p, key_at[32 * w + c], a.window, a.n_sink) ? 1u << c : 0u;
                    visible[w] = bits;
                }
            } else {
                const int past = min(p, len - 1) - j0 + 1, first = max(p - a.window + 1, 0) - j0, sink = a.n_sink - j0;
#pragma unroll
                for (int w = 0; w < kKeys / 32; ++w) visible[w] = below(past - 32 * w) & (~below(first - 32 * w) | below(sink - 32 * w));
            }
            if (a.q_pos) {                                   // (those of three tiles ago were read before the last S was made)
#pragma unroll
                for (int w = 0; w < kKeys / 32; ++w) {
                    const uint32_t any = __reduce_or_sync(0xffffffffu, visible[w]);
                    if (lane == 0) seen_by[i & 3][warp][w] = any;
                }
            }
        };
        const auto scores_there = [&](int i) { return guard.wait_all(s_full + 8 * (i & 1), i / 2 & 1); };
        const auto weigh = [&](int i) {
            const int buf = i & 1;
            if (TOKENS && twins && t >= 2 * kTwin) {
                mbar_arrive(p_full + 8 * buf);
                return true;
            }
            tc_fence_after();
            const uint32_t s_col = tmem + buf * kKeys + lanes;
            float x[kKeys];
            tmem_ld_cols<kKeys>(s_col, x);
            if (masked) {
#pragma unroll
                for (int c = 0; c < kKeys; ++c) x[c] = visible[c / 32] >> (c & 31) & 1u ? x[c] : -CUDART_INF_F;
            }
            float tops[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int c = 4; c < kKeys; c += 8) {             // (three at a time)
#pragma unroll
                for (int b = 0; b < 4; ++b) tops[b] = c + 4 + b < kKeys ? fmaxf(fmaxf(tops[b], x[c + b]), x[c + 4 + b]) : fmaxf(tops[b], x[c + b]);
            }
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * scale;      // (scale is positive)
            const bool move = top > m + kMoveAt;
            if (i > 0 && __any_sync(0xffffffffu, move)) {
                // (the step before may still be adding; the one before that was complete before this S was)
                if (!guard.wait_all(o_step, (i - 1) & 1)) return false;
                tc_fence_after();
                const float f = move ? ex2_approx(m - top) : 1.f;
#pragma unroll 1
                for (int c = 0; c < a.head_dim; c += 32) {
                    float o[32];
                    uint32_t w[32];
                    tmem_ld_cols<32>(o_col + c, o);
#pragma unroll
                    for (int k = 0; k < 32; ++k) w[k] = __float_as_uint(o[k] * f);
                    tmem_st_cols<32>(o_col + c, w);
                }
                l *= f;
            }
            if (move) m = top;
            const float ref = m == -CUDART_INF_F ? 0.f : m - kLift;
            const uint64_t ref2 = two_f32(-ref, -ref);
            uint64_t sums[2] = {0, 0};
#pragma unroll
            for (int c0 = 0; c0 < kKeys; c0 += 32) {
                uint32_t w[16];
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    float y, z;
                    split_f32(fma_f32x2(two_f32(x[c0 + c], x[c0 + c + 1]), scale2, ref2), y, z);
                    y = ex2_approx(y);
                    z = ex2_approx(z);
                    sums[c / 2 & 1] = add_f32x2(sums[c / 2 & 1], two_f32(y, z));
                    // (rounded for the product alone: the sum, which the logarithm is taken of too, is of the weights as they are.  Against 64 bits
                    // 8192 x 8192 causal is off by 2.17e-3, of which the rounding of the output to bf16 is 1.65e-3)
                    w[c / 2] = F16 ? two_f16(y, z) : two_bf16(y, z);
                    if (TOKENS && twin) w[c / 2] = two_bf16(y - __uint_as_float(w[c / 2] << 16), z - __uint_as_float(w[c / 2] & 0xFFFF0000u));
                }
                tmem_st_cols<16>(s_col + c0 / 2, w);
            }
            float even, odd;
            split_f32(add_f32x2(sums[0], sums[1]), even, odd);
            l += even + odd;
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(p_full + 8 * buf);
            return true;
        };
        bool ok = walk_tiles(0, n, 1, look, scores_there, weigh);
        // ---- the rows
        if (ok && n > 0) ok = guard.wait_all(o_full, 0);
        tc_fence_after();
        const int64_t part = s.part0 + static_cast<int64_t>(blockIdx.y) * s.n_q + i_row;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        m -= kLift;
        // the twins' rows of O, for the others (the keys and values have been read): element by element, the rows side by side
        float* const beside = reinterpret_cast<float*>(raw + (kv_at - smem_u32(raw)));
        if (TOKENS && twins && t < 2 * kTwin) {
            if (twin && ok && n > 0) {
                for (int c = 0; c < a.head_dim; c += 32) {
                    float o[32];
                    tmem_ld_cols<32>(o_col + c, o);
#pragma unroll
                    for (int k = 0; k < 32; ++k) beside[(c + k) * kTwin + r] = o[k];
                }
            }
            asm volatile("bar.sync 2, 64;" ::: "memory");    // (reached by both warps, whoever gave up)
        }
        for (int c = 0; c < a.head_dim && ok && !(TOKENS && twins && t >= kTwin); c += 32) {
            float o[32];
            if (n > 0) tmem_ld_cols<32>(o_col + c, o);
            if (TOKENS && twins && n > 0) {
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] += beside[(c + k) * kTwin + r];
            }
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
        if (mine && ok && !twin) {
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
    if (warp == Sh::kIssues) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::kColumns);
    }
}

// attend_weights_kernel: mass of 128 cached rows over the queries of their sequence, for the heads packed together.  Keys on the lanes
// of tensor memory, queries on its columns: S^T = K Q^T, and a thread adds up 2^(S - lse) over the columns of its key, so that
// no sum crosses threads.  Tiles of 128 query rows go to the two groups of four warps in turn, each with an S of its own; two CTAs to a
// multiprocessor (heads of up to 128 elements; the 96 registers that leaves spill 16 bytes: 16 frames with weights 336 us, with one CTA and no spills 378).
// Bound by the exponentials, whose pipe is busy half of the time (the tensor cores a fifth), and by the barriers between tiles.
constexpr int kWeightStages = 2;

template <int DB>
struct WeightShape {
    static constexpr int kTileBytes = DB * kRows * 128;
    static constexpr int kColumns = 2 * kRows;
    static constexpr int kSmem = 1024 + (1 + kWeightStages) * kTileBytes;
    static constexpr int kCtas = 2 * (kSmem + 6 * 1024 + kSmemReservedPerCta) <= kSmemPerSm ? 2 : 1;
};

template <bool F16, int DB>
__global__ void __launch_bounds__(kThreads, WeightShape<DB>::kCtas)
attend_weights_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap)
{
    using Sh = WeightShape<DB>;
    constexpr int ST = kWeightStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * ST + 6];
    __shared__ uint16_t list[kMaxTiles];
    __shared__ __align__(16) float row_z[2][kRows];
    __shared__ int row_p[2][kRows];
    __shared__ float half[kRows];
    __shared__ int n_list, dead;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t k_at = base, q_at = base + Sh::kTileBytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int i) { return bar0 + 8u * i; };
    const auto empty = [&](int i) { return bar0 + 8u * (ST + i); };
    const uint32_t s_full = bar0 + 8u * (2 * ST), s_empty = s_full + 16, k_full = s_full + 32, ended = s_full + 40;      // two of each group's S
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    if (warp == 8 && lane == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(s_empty + 8 * i, 128); }
        mbar_init(k_full, 1);
        mbar_init(ended, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        dead = 0;
        prefetch_tensormap(&map_q);
        prefetch_tensormap(&map_k);
    }
    __syncwarp();
    pdl_wait();
    if (warp == 9) tmem_alloc(smem_u32(&tmem_base), Sh::kColumns);
    const int packs = a.n_heads / a.pack, pk = static_cast<int>(blockIdx.x) % packs, head0 = pk * a.pack;
    const int blk = static_cast<int>(blockIdx.x) / packs;
    const AttSeq& s = a.s[seq_at(a, blk, [](const AttSeq& x) { return x.tile0; })];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack, len = seq_len(a, s), j0 = (blk - s.tile0) * kRows;
    const int q_tiles = (s.n_q + per - 1) / per;
    // the tiles of queries some of which see some of these keys: counted positions name them, else a list is made
    const Span k = a.kv_pos ? key_span(a, s, len, j0, kRows, lane) : counted_span(len, j0, kRows);
    const bool listed = a.kv_pos || a.q_pos;
    int v0 = static_cast<int>(blockIdx.y) * kMaxTiles, n = max(0, min(q_tiles - v0, kMaxTiles));
    const auto tile_flags = [&](int v) {
        int lo, hi;
        query_span(a, s, len, v * per, min((v + 1) * per, s.n_q), lane, &lo, &hi);
        const int f = span_flags(a, lo, hi, k);
        return f && ((v + 1) * per > s.n_q || per * a.pack < kRows) ? f | kMask : f;
    };
    if (listed) {
        for (int v = warp; v < n; v += kThreads / 32) {
            const int f = tile_flags(v0 + v);
            if (lane == 0) list[v] = static_cast<uint16_t>(f);
        }
        __syncthreads();
        if (warp == 0) {
            const int c = compact_entries(list, n, lane);
            if (lane == 0) n_list = c;
        }
        __syncthreads();
        n = n_list;
    } else {
        // queries from the first key's position on, up to the last one whose window reaches the last key (any, where a sink is among them)
        const int p0 = len - s.n_q, last = v0 + n;
        const int from = max(k.lo - p0, 0) / per;
        const int64_t reach = k.lo < a.n_sink ? s.n_q : min(static_cast<int64_t>(k.hi) - p0 + a.window, static_cast<int64_t>(s.n_q));
        const int to = k.hi < 0 || reach <= 0 ? 0 : static_cast<int>((reach + per - 1) / per);
        const int first = max(v0, min(from, last));
        n = max(0, min(to, last) - first);
        v0 = first;
    }
    const auto tile_at = [&](int i) { return v0 + (listed ? list[i] >> kEntryShift : i); };
    Guard guard = {&dead, a.status};
    const auto load = [&](int c) {
        const int st = c % ST, row = s.qm_row + tile_at(c) * per;
        mbar_expect_tx(full(st), DB * per * a.pack * 128);
        for (int i = 0; i < DB; ++i) tma_load_3d(q_at + st * Sh::kTileBytes + i * kRows * 128, &map_q, i * 64, head0, row, full(st));
    };
    const int at_once = min(ST, n);
    if (warp == 8 && lane == 0 && n > 0) {
        mbar_expect_tx(k_full, Sh::kTileBytes);
        for (int i = 0; i < DB; ++i) tma_load_3d(k_at + i * kRows * 128, &map_k, i * 64, hk, s.km_row + j0, k_full);
        for (int c = 0; c < at_once; ++c) load(c);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base;

    if (warp == 8) {
        if (n > 0 && lane == 0) {
            int c = at_once;
            for (; c < n; ++c) {
                if (!guard.wait(empty(c % ST), (c / ST - 1) & 1)) break;
                load(c);
            }
            guard.settle(k_full, 0);
            for (int i = max(0, c - ST); i < c; ++i) guard.settle(full(i % ST), i / ST & 1);
        }
    } else if (warp == 9) {
        const uint32_t idesc = idesc_16<F16>(kRows);
        const int steps = a.head_dim / 16;
        const bool one = elect_one();
        bool ok = n == 0 || guard.wait_all(k_full, 0);
        for (int i = 0; i < n && ok; ++i) {
            const int st = i % ST, buf = i & 1;
            ok = guard.wait_all(full(st), i / ST & 1) && (i < 2 || guard.wait_all(s_empty + 8 * buf, (i / 2 - 1) & 1));
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
        if (one) umma_commit(ended);
        __syncwarp();
        guard.settle(ended, 0);
    } else {
        const int group = warp / 4, r = t & 127, j = j0 + r;
        const uint32_t s_col = tmem + group * kRows + (static_cast<uint32_t>(warp & 3) << 21);
        const int c_pos = key_pos(a, s, len, j);
        const uint64_t scale2 = two_f32(a.scale_log2, a.scale_log2);
        float sum = 0.f;
        // this thread's query row of a tile, for all keys of the group: logarithm of its sum, position
        float z = 0.f;
        int p = -1;
        const auto fetch = [&](int i) {
            const int iq = i < n ? tile_at(i) * per + r / a.pack : s.n_q;
            const bool there = r < per * a.pack && iq < s.n_q;
            z = there ? a.lse2[static_cast<int64_t>(s.qp0 + iq) * a.n_heads + head0 + r % a.pack] : 0.f;
            p = there ? query_pos(a, s, len, iq) : -1;
        };
        fetch(group);
        bool masked = false;
        uint32_t visible[kRows / 32];                        // a bit for every query row that sees this thread's key
        const auto look = [&](int i) {
            asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");       // (nobody reads the last tile's any more)
            row_z[group][r] = -z;
            row_p[group][r] = p;
            asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
            fetch(i + 2);
            const int v = tile_at(i);
            masked = listed ? (list[i] & kMask) != 0 : tile_flags(v) != kNeed;
            if (masked) {
                if (listed) {
#pragma unroll
                    for (int w = 0; w < kRows / 32; ++w) {
                        uint32_t bits = 0;
#pragma unroll 8
                        for (int c = 0; c < 32; ++c) bits |= sees(row_p[group][32 * w + c], c_pos, a.window, a.n_sink) ? 1u << c : 0u;
                        visible[w] = bits;
                    }
                } else {
                    const int q0 = len - s.n_q + v * per, there = min(per, s.n_q - v * per);      // position of the tile's first query, and how many
                    const int first = max(c_pos - q0, 0), past = c_pos < 0 ? 0 : c_pos < a.n_sink ? there : static_cast<int>(min(static_cast<int64_t>(c_pos) - q0 + a.window, static_cast<int64_t>(there)));
#pragma unroll
                    for (int w = 0; w < kRows / 32; ++w)
                        visible[w] = below(max(past, 0) * a.pack - 32 * w) & ~below(min(first, per) * a.pack - 32 * w);
                }
            }
        };
        const auto scores_there = [&](int i) { return guard.wait_all(s_full + 8 * group, i / 2 & 1); };
        const auto add_up = [&](int) {
            tc_fence_after();
            uint64_t part[2] = {0, 0};
#pragma unroll
            for (int c0 = 0; c0 < kRows; c0 += 32) {
                float x[32];
                tmem_ld_cols<32>(s_col + c0, x);
                if (c0 + 32 == kRows) {                      // S is read: the next one may come
                    tc_fence_before();
                    mbar_arrive(s_empty + 8 * group);
                }
#pragma unroll
                for (int c = 0; c < 32; c += 4) {            // (row_z: what the logarithms of the sums take off)
                    const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(&row_z[group][c0 + c]);
                    split_f32(fma_f32x2(two_f32(x[c], x[c + 1]), scale2, y.x), x[c], x[c + 1]);
                    split_f32(fma_f32x2(two_f32(x[c + 2], x[c + 3]), scale2, y.y), x[c + 2], x[c + 3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[c + e] = ex2_approx(x[c + e]);
                }
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) x[c] = visible[c0 / 32] >> c & 1u ? x[c] : 0.f;
                }
#pragma unroll
                for (int c = 0; c < 32; c += 2) part[c / 2 & 1] = add_f32x2(part[c / 2 & 1], two_f32(x[c], x[c + 1]));
            }
            float even, odd;
            split_f32(add_f32x2(part[0], part[1]), even, odd);
            sum += even + odd;
            return true;
        };
        walk_tiles(group, n, 2, look, scores_there, add_up);
        if (group == 1) half[r] = sum;
        asm volatile("bar.sync 3, 256;" ::: "memory");
        if (group == 0 && j < s.n_kv)
            a.part_mass[(static_cast<int64_t>(blockIdx.y) * packs + pk) * a.total_kv + s.kvp0 + j] = sum + half[r];
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::kColumns);
    }
}

template <class K>
cudaError_t launch(KernelSetup& setup, K kernel, dim3 grid, int threads, int columns, size_t smem, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    smem = smem_for_tmem(smem, columns);                     // (no CTA more than there is tensor memory for)
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(kernel), smem, columns);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, maps.q, maps.k, maps.v);
}

template <bool F16, int DB, bool TOKENS>
cudaError_t attend(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    static KernelSetup setup;
    const dim3 grid(static_cast<unsigned>(a.n_blocks) * static_cast<unsigned>(a.n_heads / a.pack), static_cast<unsigned>(a.splits));
    using Sh = TileShape<DB>;
    return launch(setup, attend_tile_kernel<F16, DB, TOKENS>, grid, Sh::kWarps * 32, Sh::kColumns, Sh::kSmem, a, maps, stream);
}

template <bool F16, int DB>
cudaError_t weights(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    static KernelSetup setup;
    const AttSeq& last = a.s[a.n_seq - 1];
    const int64_t tiles = last.tile0 + (last.n_kv + kRows - 1) / kRows;
    if (tiles == 0) return cudaSuccess;
    const int packs = a.n_heads / a.pack;
    return launch(setup, attend_weights_kernel<F16, DB>, dim3(static_cast<unsigned>(tiles * packs), static_cast<unsigned>(a.mass_parts / packs)), kThreads,
                  WeightShape<DB>::kColumns, WeightShape<DB>::kSmem, a, maps, stream);
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
template <bool F16, bool TOKENS>
cudaError_t attend_by_dim(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    switch ((a.head_dim + 63) / 64) {
    case 1: return attend<F16, 1, TOKENS>(a, maps, stream);
    case 2: return attend<F16, 2, TOKENS>(a, maps, stream);
    case 3: return attend<F16, 3, TOKENS>(a, maps, stream);
    default: return attend<F16, 4, TOKENS>(a, maps, stream);
    }
}
}  // namespace

cudaError_t launch_attend_weights(bool f16, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    return f16 ? weights_by_dim<true>(a, maps, stream) : weights_by_dim<false>(a, maps, stream);
}

cudaError_t launch_attend_tile(bool f16, bool tokens, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    if (f16) return attend_by_dim<true, false>(a, maps, stream);
    return tokens ? attend_by_dim<false, true>(a, maps, stream) : attend_by_dim<false, false>(a, maps, stream);
}

}  // namespace mvla
