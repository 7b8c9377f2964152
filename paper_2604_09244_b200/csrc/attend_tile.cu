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
#include "attend_tile.cuh"
#include "attend_walk.h"

#include <cuda_fp16.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 320;                // attend_weights_kernel
constexpr float kLargeScore = 65536.f;       // beyond, scores over pages are not scaled and taken from their reference in one step
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

// PAGED: keys and values lie in pages (a tile is the rows of one, or of several side by side), positions are counted, and every sequence is cut into parts
// of its own number: a.n_blocks counts its blocks of queries times its parts.  A part is a cluster's, whose CTAs join their sums through shared memory.
template <bool F16, int DB, bool TOKENS, bool PAGED>
__global__ void __launch_bounds__(TileShape<DB>::kWarps * 32, TileShape<DB>::kCtas)
attend_tile_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v)
{
    using Sh = TileShape<DB>;
    constexpr int ST = Sh::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 8];
    __shared__ __align__(16) uint16_t list[kMaxTiles];
    static_assert(sizeof list >= 4 * kJoinFloats, "room for the factors of a cluster's rows");
    __shared__ int key_at[kKeys];
    __shared__ uint32_t seen_by[4][4][kKeys / 32];           // of the last tiles: the keys that some row of a warp sees
    __shared__ int n_list, dead;
    __shared__ uint32_t tmem_base;
    __shared__ float2 row_ml[PAGED ? kRows : 1];
    static_assert(ST * Sh::kStage >= DB * 64 * kRows * 4, "room for the sums of a cluster's CTA");
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
    const int ranks = PAGED ? cluster_ctas() : 1, cta = static_cast<int>(blockIdx.x) / ranks;
    const int heads = a.n_heads / a.pack, blk = a.n_blocks - 1 - cta / heads, head0 = cta % heads * a.pack;
    const AttSeq& s = a.s[seq_of_block(a, blk)];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack;      // queries of the tile
    const int part_of_seq = PAGED ? (blk - s.blk0) % s.parts : static_cast<int>(blockIdx.y);       // (pages: a cluster's)
    const int parts = PAGED ? s.parts * ranks : a.splits, piece = PAGED && ranks > 1 ? part_of_seq * ranks + static_cast<int>(cluster_ctarank()) : part_of_seq;
    const int q0 = (PAGED ? (blk - s.blk0) / s.parts : blk - s.blk0) * per, len = seq_len(a, s);
    const bool twins = TOKENS && static_cast<int64_t>(s.n_q) * (a.n_heads / a.kv_heads) <= kTokenRows;
    int lo, hi;
    query_span(a, s, len, q0, min(q0 + per, s.n_q), lane, &lo, &hi);
    const TileRange range = tile_range(a, len, lo, hi, kKeys);
    const int per_split = (range.count + parts - 1) / parts, v0 = piece * per_split;
    int n = max(0, min(range.count - v0, per_split));
    if (!PAGED && a.kv_pos) {
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
    const auto first_key = [&](int i) { return range.tile(v0 + (!PAGED && a.kv_pos ? list[i] >> kEntryShift : i)) * kKeys; };
    const auto flags_of = [&](int i, int j0) {
        if (!PAGED && a.kv_pos) return static_cast<int>(list[i]);
        const Span k = counted_span(len, j0, kKeys);
        const int f = span_flags(a, lo, hi, k);              // (queries far apart may leave out a tile between them: then no row sees a key)
        return f ? f : kMask;
    };
    Guard guard = {&dead, a.status};

    // ---- loads (one lane of a warp; with pages a lane to every box, which looks its page up a tile ahead): the first ones before the CTA meets
    const int box_rows = PAGED ? min(kKeys, 1 << a.page_shift) : kKeys, boxes = DB * (kKeys / box_rows);
    const int row_of_box = lane / DB * box_rows, piece_of_box = lane % DB;
    const TileRange whole = PAGED && !a.table ? tile_range(a, len, query_pos(a, s, len, 0), query_pos(a, s, len, s.n_q - 1), kKeys) : TileRange{0, 0, 0};
    const auto look_up = [&](int i) {                        // where this lane's box of tile i lies: outside the map where there is nothing (zeros)
        if (!PAGED || lane >= boxes || i >= n) return -1;
        const int j = first_key(i) + row_of_box, tile = j / kKeys;
        if (!a.table) return (s.km_row + (tile < whole.sinks ? tile : tile - whole.first + whole.sinks)) * a.kv_heads + hk;      // (seen tiles, one after another)
        const int page = j < len ? a.table[s.index * a.table_stride + (j >> a.page_shift)] : -1;
        return page >= 0 && page < a.n_pages ? page * a.kv_heads + hk : -1;
    };
    int here = 0, ahead = 0;
    const auto load_box = [&](int c) {                       // (pages: this lane's box of chunk c, on page `here`)
        const int st = c % ST, j0 = first_key(c / 2);
        const CUtensorMap* const map = c & 1 ? &map_v : &map_k;
        if constexpr (!PAGED) {
            mbar_expect_tx(full(st), Sh::kStage);
            for (int b = 0; b < DB; ++b) tma_load_3d(kv_at + st * Sh::kStage + b * kKeys * 128, map, b * 64, hk, s.km_row + j0, full(st));
        } else {
            if (lane == 0) mbar_expect_tx(full(st), Sh::kStage);
            __syncwarp();
            if (lane < boxes)
                tma_load_3d(kv_at + st * Sh::kStage + piece_of_box * kKeys * 128 + row_of_box * 128, map, piece_of_box * 64,
                            (j0 + row_of_box) & ((1 << a.page_shift) - 1), here, full(st));
        }
    };
    const auto load = [&](int c) {                           // tiles of keys and values in turn
        if (PAGED && !(c & 1)) {
            here = ahead;
            ahead = look_up(c / 2 + 1);
        }
        load_box(c);
    };
    const int at_once = min(ST, 2 * n);
    if (warp == Sh::kLoads && (PAGED || lane == 0) && n > 0) {
        if (lane == 0) {
            mbar_expect_tx(q_full, DB * per * a.pack * 128);
            for (int b = 0; b < DB; ++b) tma_load_3d(q_at + b * kRows * 128, &map_q, b * 64, head0, s.qm_row + q0, q_full);
        }
        if constexpr (PAGED) {                               // (the pages of the first tiles, all at once)
            int pages[(ST + 1) / 2 + 1];
#pragma unroll
            for (int i = 0; i <= (ST + 1) / 2; ++i) pages[i] = look_up(i);
#pragma unroll
            for (int c = 0; c < ST; ++c)
                if (c < at_once) {
                    here = pages[c / 2];
                    load_box(c);
                }
            ahead = pages[(ST + 1) / 2];
        } else {
            for (int c = 0; c < at_once; ++c) load(c);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base;

    if (warp == Sh::kLoads) {
        int c = at_once;
        if (PAGED && n > 0) {
            for (; c < 2 * n; ++c) {
                if (!guard.wait_all(empty(c % ST), (c / ST - 1) & 1)) break;
                load(c);
            }
        }
        if (lane == 0 && n > 0) {
            if (!PAGED) {
                for (; c < 2 * n; ++c) {
                    if (!guard.wait(empty(c % ST), (c / ST - 1) & 1)) break;
                    load(c);
                }
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
                if (!PAGED && a.q_pos) {
                    ok = guard.wait_all(p_full + 8 * (i & 1), i / 2 & 1);
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int x = 0; x < kKeys / 32; ++x) by[x] |= seen_by[i & 3][w][x];
                }
                bool some = false;
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x) {
                    const int k = 32 * x + lane;
                    if (!PAGED && a.q_pos ? by[x] >> lane & 1u : j0 + k < len && some_sees(lo, hi, j0 + k, a.window, a.n_sink)) continue;
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
            if (!PAGED && a.kv_pos) {                        // the positions, for the four warps
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
            if (!PAGED && a.q_pos) {                         // (those of three tiles ago were read before the last S was made)
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
            const float top = __fmul_rn(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), scale);      // (scale is positive; rounded before anything is taken from it)
            const bool move = PAGED ? top - m > kMoveAt : top > m + kMoveAt;
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
            uint64_t by2 = scale2, ref2 = two_f32(-ref, -ref);
            if (PAGED && fabsf(ref) > kLargeScore) {         // (the largest score's distance from its reference is nothing, however large: rounded as that was.  A row by itself: some are nobody's)
#pragma unroll
                for (int c = 0; c < kKeys; ++c) x[c] = __fadd_rn(__fmul_rn(x[c], scale), -ref);
                by2 = two_f32(1.f, 1.f);
                ref2 = 0;
            }
            uint64_t sums[2] = {0, 0};
#pragma unroll
            for (int c0 = 0; c0 < kKeys; c0 += 32) {
                uint32_t w[16];
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    float y, z;
                    split_f32(fma_f32x2(two_f32(x[c0 + c], x[c0 + c + 1]), by2, ref2), y, z);
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
        const int64_t part = s.part0 + static_cast<int64_t>(part_of_seq) * s.n_q + i_row;
        const bool joined = PAGED && ranks > 1, split = PAGED ? s.parts > 1 : a.splits > 1;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        m -= kLift;
        float4* const sums = reinterpret_cast<float4*>(raw + (kv_at - smem_u32(raw)));      // of a cluster's CTA (sums_at)
        // the twins' rows of O, for the others (the keys and values have been read): element by element, the rows side by side
        float* const beside = reinterpret_cast<float*>(raw + ((PAGED ? q_at : kv_at) - smem_u32(raw)));
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
            for (int k = 0; k < 32; ++k) o[k] = l > 0.f ? (joined || split ? o[k] : o[k] * inv) : 0.f;
            if (joined) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) sums[sums_at(t, (c + k) / 4, a.head_dim)] = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                continue;
            }
            if (!mine) continue;
            if (split) {
                float* const dst = a.part_o + (part * a.n_heads + head) * a.head_dim + c;
#pragma unroll
                for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            } else {
                __nv_bfloat16* const dst = static_cast<__nv_bfloat16*>(a.out) + ((s.q_row + i_row) * a.n_heads + head) * a.head_dim + c;
#pragma unroll
                for (int k = 0; k < 32; k += 8) store8(dst + k, o + k);
            }
        }
        if (joined) row_ml[t] = make_float2(m, l);
        if (mine && ok && !twin && !joined) {
            if (split) {
                a.part_ml[part * a.n_heads + head] = make_float2(m, l);
            } else {
                const float z = l > 0.f ? m + log2f(l) : -CUDART_INF_F;
                if (a.lse) a.lse[(s.q_row + i_row) * a.n_heads + head] = z * 0.69314718055994531f;      // ln 2
                if (!PAGED && a.mass) a.lse2[static_cast<int64_t>(s.qp0 + i_row) * a.n_heads + head] = z;
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    // (before the cluster meets: who holds tensor memory waits for no other CTA, which may wait for some of it behind another launch's)
    if (warp == Sh::kIssues) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::kColumns);
    }
    if (PAGED && ranks > 1) {                                // (reached by all CTAs of the cluster, whoever gave up)
        cluster_arrive_release();
        cluster_wait_acquire();
        join_cluster<1>(a, s, kv_at, smem_u32(row_ml), reinterpret_cast<float*>(list), ranks, q0, per, head0, part_of_seq);      // (no list of counted positions)
        cluster_arrive_release();                            // (nobody's sums are gone while another reads them)
        cluster_wait_acquire();
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
cudaError_t launch(KernelSetup& setup, K kernel, dim3 grid, int threads, int columns, size_t smem, const AttArgs& a, const AttMaps& maps, cudaStream_t stream, int cluster = 1)
{
    smem = smem_for_tmem(smem, columns);                     // (no CTA more than there is tensor memory for)
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(kernel), smem, columns);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, maps.q, maps.k, maps.v);
}

template <bool F16, int DB, bool TOKENS, bool PAGED>
cudaError_t attend(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    static KernelSetup setup;
    const int cluster = PAGED ? a.cluster : 1;
    const dim3 grid(static_cast<unsigned>(a.n_blocks) * static_cast<unsigned>(a.n_heads / a.pack) * static_cast<unsigned>(cluster), PAGED ? 1u : static_cast<unsigned>(a.splits));
    using Sh = TileShape<DB>;
    return launch(setup, attend_tile_kernel<F16, DB, TOKENS, PAGED>, grid, Sh::kWarps * 32, Sh::kColumns, Sh::kSmem, a, maps, stream, cluster);
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
template <bool F16, bool TOKENS, bool PAGED>
cudaError_t attend_by_dim(const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    switch ((a.head_dim + 63) / 64) {
    case 1: return attend<F16, 1, TOKENS, PAGED>(a, maps, stream);
    case 2: return attend<F16, 2, TOKENS, PAGED>(a, maps, stream);
    case 3: return attend<F16, 3, TOKENS, PAGED>(a, maps, stream);
    default: return attend<F16, 4, TOKENS, PAGED>(a, maps, stream);
    }
}
}  // namespace

cudaError_t launch_attend_weights(bool f16, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    return f16 ? weights_by_dim<true>(a, maps, stream) : weights_by_dim<false>(a, maps, stream);
}

cudaError_t launch_attend_tile(bool f16, bool tokens, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    if (f16) return attend_by_dim<true, false, false>(a, maps, stream);
    return tokens ? attend_by_dim<false, true, false>(a, maps, stream) : attend_by_dim<false, false, false>(a, maps, stream);
}

cudaError_t launch_page_tile(bool tokens, const AttArgs& a, const AttMaps& maps, cudaStream_t stream)
{
    return tokens ? attend_by_dim<false, true, true>(a, maps, stream) : attend_by_dim<false, false, true>(a, maps, stream);
}

}  // namespace mvla
