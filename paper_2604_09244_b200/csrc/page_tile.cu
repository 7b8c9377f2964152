// Attention of chunks of new tokens over quantised pages on the tensor cores: keys and values are unpacked to fp16 on their way into shared memory.
//
// As attend_tile.cu: a CTA has a tile of 128 query rows that share a key head and walks the tiles of 64 keys of its part,
//     S = Q K^T  ->  P = 2^(S - reference) in fp16, back into the columns of S  ->  O += P V,
// a thread to a row in the softmax (warps 0-3), S double-buffered, one warp that issues the MMAs.  A warp copies codes and scales into a ring, what a tile has of
// a page at a time; four warps turn them into fp16 and store them as the MMAs read them (128-byte swizzle).
// Scales are powers of two.  A tile's largest scale of its keys becomes a factor of its scores and the largest one of its values a factor of its weights (both the same
// for the whole tile); what a row, or 32 elements, have less is multiplied into the codes, which have as much room above in fp16 (2^7 for e4m3, 2^13 for e2m1) and keep their bits down to 2^-24.  Where
// the scales of a tile lie further apart (kKeySpread, kSpread), codes are taken against their own row's largest scale (groups below 2^-27 of it count as nothing), which becomes a factor of that row's
// scores, or part of its weights (two exponentials to a key): what other queries see takes no bits.  The products of weights and scales that make up a row's output are of other sizes than its
// weights, so that they have a reference of their own, in which O is counted.  Queries are fp16 too, every row times a power of two that puts its largest element between 2^14 and 2^15.
//
// A CTA has one tile of query rows (two CTAs to a multiprocessor, heads of up to 128 elements; 96 registers, 44 bytes spill), or two that share what is unpacked (one CTA); the softmax reads S
// twice, once for its maximum.  B200, 32 query heads over 8 heads of 128, e4m3: 5 tokens over 60000 rows 63 us, 4 chunks of 56 over 3100 to 5500 rows 49 (one tile of rows to a CTA: 54), of 33
// over 4000 rows 40 (48).  Two tiles of rows and 64 keys take 1.8 us, about as in attend_tile.cu: without the exponentials, without most of the unpacking or of the second product 0 to 10 % less, so that it
// is the way of a tile from warp to warp.  The codes a tile ahead in registers instead of a ring: half as long again (a warp's loads wait for one another); twice the ring: the same.
// The 4 chunks with all keys' scales far apart 61 us, with all values' 80 (unpacked first, whatever the scales, 58): such tiles are taken for rare ones.
#include "attend_tile.cuh"
#include "attend_walk.h"
#include "page.cuh"

#include <algorithm>
#include <cfloat>

namespace mvla {
namespace {

template <int KIND> struct Codes;
template <> struct Codes<MVLA_PAGE_E4M3> { using Word = uint2; static constexpr int kLift = 7; };       // eight elements; room above the codes in fp16
template <> struct Codes<MVLA_PAGE_E2M1> { using Word = uint32_t; static constexpr int kLift = 13; };

// T: tiles of 128 query rows to a CTA, which share what is unpacked: one and two CTAs to a multiprocessor (heads of up to 128 elements), or two and one CTA.
template <int KIND, int D32, int T>
struct PageTileShape {
    static constexpr int kDB = (D32 + 1) / 2;                // boxes of 64 elements
    static constexpr int kIssues = 4 * T, kLoads = kIssues + 1, kDecodes = kIssues + 2, kDecoders = 4, kWarps = kDecodes + kDecoders;
    static constexpr int kO = 2 * kKeys, kOf = kO + kDB * 64;       // columns of tensor memory of a tile of rows: S (two buffers, P in the same columns), then O
    static constexpr int kColumns = T * kOf <= 256 ? 256 : 512;
    static_assert(T * kOf <= kTmemColsPerSm, "shape");
    static constexpr int kCtas = T == 1 ? kTmemColsPerSm / kColumns : 1;
    static constexpr int kQBytes = T * kDB * kRows * 128, kStage = kDB * kKeys * 128;
    // the ring: codes of a tile's keys, with the scales of its keys and values, or codes of its values
    static constexpr int kRowBytes = page_row_bytes(KIND, D32 * 32, 2), kGroups = page_row_scales(KIND, D32 * 32);
    static constexpr int kCodes = kKeys * kRowBytes, kSlot = kCodes + 2 * kKeys * kGroups, kSlots = T == 1 ? 3 : 4;
    static constexpr int kFixed = (T == 2 ? 8 : KIND == MVLA_PAGE_E4M3 ? 6 : 9) * 1024;      // static shared memory, and what the tiles' alignment takes
    static constexpr int kRoom = ((kCtas == 2 ? kSmemPerSm / 2 - kSmemReservedPerCta : kSmemMaxPerCta) - kFixed - kQBytes - kSlots * kSlot) / kStage;
    static constexpr int kStages = kRoom > kMaxStages ? kMaxStages : kRoom;
    static constexpr int kSmem = 1024 + kQBytes + kStages * kStage + kSlots * kSlot;
    static constexpr int kPieces = 8 * D32 / kDecoders;      // of eight elements, of a decoding thread, in a tile of keys or of values
    static_assert(kStages >= 3 && kSlot % 16 == 0, "shape");
};
// Of a tile, for the softmax: of every row of values the exponent of its scale, the largest and the least of them; of every row of keys that exponent, and the largest; which of the two are far apart.
constexpr int kFarValues = 1, kFarKeys = 2;
struct __align__(16) TileScales {
    float exponent[kKeys];
    int key[kKeys];
    float most, least;
    int most_key, far;
};
// The reference of weights times scales is the largest one, or (where a tile's are not far apart) at most 2^kSpread below; against the tile's largest scale no weight is more than 2^kMoveAt
// above the reference, and with its own, which counts where they are far apart, none either: 2^(kMoveAt + kF16Lift) is a number of fp16.
constexpr int kSpread = 6;
template <int KIND> constexpr int kKeySpread = KIND == MVLA_PAGE_E4M3 ? 21 : 9;
constexpr float kMoveScaledAt = kMoveAt - kSpread;
constexpr float kLargeScore = 1024.f;        // beyond, scores and exponents of scales are not added up in one number (2^-13 of a weight is lost so), nor scores scaled and taken from their reference in one step
constexpr int kTileScales = 4;               // tiles whose scales are kept

__device__ __forceinline__ void codes_f16(uint2 w, uint32_t (&h)[4])
{
    from_e4m3(w.x, h[0], h[1]);
    from_e4m3(w.y, h[2], h[3]);
}
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t (&h)[4]) { from_e2m1(w, h); }
__device__ __forceinline__ uint32_t times2(uint32_t x, uint32_t f)
{
    const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&f));
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Bits of 2^e in fp16, e at most 15: below 2^-24 zero.
__device__ __forceinline__ uint32_t power_f16(int e) { return e > -15 ? static_cast<uint32_t>(e + 15) << 10 : e >= -24 ? 1u << (e + 24) : 0u; }
__device__ __forceinline__ void store16(uint32_t at, const uint32_t (&w)[4])
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
// What few tiles need, out of the way of the others (inside the loop over tiles it costs every one of them: 5 of 48 us).  Of this thread's row of S at `s_col`; `sees`: a bit to every key.
__device__ __forceinline__ void load_scores(uint32_t s_col, uint32_t sees, float (&x)[32])
{
    tmem_ld_cols<32>(s_col, x);
#pragma unroll
    for (int c = 0; c < 32; ++c) x[c] = sees >> c & 1u ? x[c] : -CUDART_INF_F;
}
// fraction 2^(key - lifted), a normal number, whatever the sizes: zero times the -infinity of a row that is not seen is no number; scores that small are as good as zero, and larger ones are beyond 32 bits.
__device__ __forceinline__ float score_scale(float fraction, int key, int lifted) { return fraction * two_to(min(max(key - lifted, -126), 127)); }
// Every key's own scale: the scores as they are, in place.
__device__ __noinline__ void scale_scores(uint32_t s_col, const int* key, float fraction, int lifted)
{
#pragma unroll 1
    for (int c0 = 0; c0 < kKeys; c0 += 32) {
        float x[32];
        uint32_t y[32];
        tmem_ld_cols<32>(s_col + c0, x);
#pragma unroll
        for (int c = 0; c < 32; ++c) y[c] = __float_as_uint(x[c] * score_scale(fraction, key[c0 + c], lifted));
        tmem_st_cols<32>(s_col + c0, y);
    }
    tmem_st_wait();
}
// The largest weight times scale, from the scores' reference on: what other queries see does not count.
__device__ __noinline__ float top_product(uint32_t s_col, uint32_t sees0, uint32_t sees1, const float* exponent, float scale, float ref)
{
    float top = -CUDART_INF_F;
#pragma unroll 1
    for (int c0 = 0; c0 < kKeys; c0 += 32) {
        float x[32];
        load_scores(s_col + c0, c0 ? sees1 : sees0, x);
#pragma unroll
        for (int c = 0; c < 32; ++c) top = fmaxf(top, __fadd_rn(__fmul_rn(x[c], scale), -ref) + exponent[c0 + c]);
    }
    return top;
}
// The weights with their rows' scales (`exponent`, null: `most`), against `above` the scores' reference, in fp16 in the columns of S; returns the sum of those without.  (The largest score's distance from its
// reference, however large they are, is nothing: rounded as that was.)
__device__ __noinline__ float weigh_far(uint32_t s_col, uint32_t sees0, uint32_t sees1, const float* exponent, float most, float scale, float ref, float above)
{
    float sum = 0.f;
#pragma unroll 1
    for (int c0 = 0; c0 < kKeys; c0 += 32) {
        float x[32];
        uint32_t weights[16];
        load_scores(s_col + c0, c0 ? sees1 : sees0, x);
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
            const float2 e = exponent ? *reinterpret_cast<const float2*>(exponent + c0 + c) : make_float2(most, most);
            const float y = __fadd_rn(__fmul_rn(x[c], scale), -ref), z = __fadd_rn(__fmul_rn(x[c + 1], scale), -ref);
            sum += ex2_approx(y + kF16Lift) + ex2_approx(z + kF16Lift);
            weights[c / 2] = two_f16(ex2_approx(y + (e.x - above + kF16Lift)), ex2_approx(z + (e.y - above + kF16Lift)));
        }
        tmem_st_cols<16>(s_col + c0 / 2, weights);
    }
    return sum;
}
// Where eight elements of a row lie in a tile of such rows, in boxes of 64 elements of `rows` rows.
__device__ __forceinline__ uint32_t swizzled(int row, int piece, int rows) { return piece / 8 * rows * 128 + row * 128 + ((piece & 7) ^ (row & 7)) * 16; }

template <int KIND, int D32, int T>
__global__ void __launch_bounds__(PageTileShape<KIND, D32, T>::kWarps * 32, PageTileShape<KIND, D32, T>::kCtas)
page_tile_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ PagePool pool)
{
    using Sh = PageTileShape<KIND, D32, T>;
    using Word = typename Codes<KIND>::Word;
    constexpr bool kE2m1 = KIND == MVLA_PAGE_E2M1;
    constexpr int D = D32 * 32, ST = Sh::kStages, P = Sh::kPieces, G = kE2m1 ? D32 : 1, kCodeLift = Codes<KIND>::kLift, kRowBytes = Sh::kRowBytes;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 3 + 5 * T + 2 * Sh::kSlots];
    __shared__ unsigned groups_there[Sh::kSlots];            // of a slot: a bit to every 16 rows that have a page
    __shared__ uint32_t factors[2][kKeys][G];                // of a tile's keys and values: fp16, twice
    __shared__ uint2 warp_top[4];                            // largest and least byte of 32 rows' scales
    __shared__ TileScales scales[kTileScales];
    __shared__ int dead;
    __shared__ uint32_t tmem_base;
    __shared__ float2 row_ml[T][kRows];
    static_assert(sizeof bars + sizeof factors + sizeof scales + sizeof row_ml + 128 + 1024 <= Sh::kFixed, "room beside the tiles");
    static_assert(Sh::kSmem - 1024 >= T * (D * kRows + kJoinFloats) * 4, "room for the sums of a cluster's CTA");
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, kv_at = base + Sh::kQBytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int i) { return bar0 + 8u * i; };
    const auto empty = [&](int i) { return bar0 + 8u * (kMaxStages + i); };
    const uint32_t q_full = bar0 + 8u * (2 * kMaxStages), o_full = q_full + 8, ended = q_full + 16, first = q_full + 24;
    // of tile `w` of rows, of S buffer `buf`
    const auto s_full = [&](int w, int buf) { return first + 8u * (5 * w + buf); };
    const auto p_full = [&](int w, int buf) { return first + 8u * (5 * w + 2 + buf); };
    const auto o_step = [&](int w) { return first + 8u * (5 * w + 4); };
    const uint32_t ring_at = kv_at + ST * Sh::kStage;
    const uint8_t* const ring = raw + (ring_at - smem_u32(raw));
    const auto raw_full = [&](int i) { return first + 8u * (5 * T + i); };
    const auto raw_empty = [&](int i) { return first + 8u * (5 * T + Sh::kSlots + i); };
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;

    if (warp == Sh::kIssues && lane == 0) {
        for (int i = 0; i < ST; ++i) { mbar_init(full(i), Sh::kDecoders); mbar_init(empty(i), 1); }
        mbar_init(q_full, 4 * T);
        for (int w = 0; w < T; ++w) {
            for (int i = 0; i < 2; ++i) { mbar_init(s_full(w, i), 1); mbar_init(p_full(w, i), 128); }
            mbar_init(o_step(w), 1);
        }
        mbar_init(o_full, 1);
        mbar_init(ended, 1);
        for (int i = 0; i < Sh::kSlots; ++i) { mbar_init(raw_full(i), 1); mbar_init(raw_empty(i), Sh::kDecoders); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        dead = 0;
    }
    __syncwarp();
    pdl_wait();
    // (only now: what holds tensor memory ahead of this kernel in the stream is complete, and nothing that holds some waits for this CTA)
    if (warp == Sh::kIssues) tmem_alloc(smem_u32(&tmem_base), Sh::kColumns);
    const int ranks = cluster_ctas(), cta = static_cast<int>(blockIdx.x) / ranks;
    const int heads = a.n_heads / a.pack, blk = a.n_blocks - 1 - cta / heads, head0 = cta % heads * a.pack;
    const AttSeq& s = a.s[seq_of_block(a, blk)];
    const int hk = head0 / (a.n_heads / a.kv_heads), per = kRows / a.pack;      // queries of the tile
    const int part_of_seq = (blk - s.blk0) % s.parts, parts = s.parts * ranks, piece_of_seq = ranks > 1 ? part_of_seq * ranks + static_cast<int>(cluster_ctarank()) : part_of_seq;
    const int q0 = (blk - s.blk0) / s.parts * (T * per), len = seq_len(a, s);
    const int lo = query_pos(a, s, len, q0), hi = query_pos(a, s, len, min(q0 + T * per, s.n_q) - 1);
    const TileRange range = tile_range(a, len, lo, hi, kKeys);
    const int per_part = (range.count + parts - 1) / parts, v0 = piece_of_seq * per_part, n = max(0, min(range.count - v0, per_part));
    const auto first_key = [&](int i) { return range.tile(v0 + i) * kKeys; };
    const auto masks = [&](int j0) {                         // whether some row does not see some key of a tile
        return span_flags(a, lo, hi, counted_span(len, j0, kKeys)) != kNeed;
    };
    Guard guard = {&dead, a.status};

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base;

    if (warp == Sh::kLoads) {
        // ---- codes and scales: chunk 2 i the keys of tile i and both scales, chunk 2 i + 1 its values; a lane to every 16 rows, of which the first of a page copies
        // what the tile has of it (4 chunks of 56: 16 rows at a time, and from pages of 16, 51.5 us, 64 rows 48)
        const int rows = min(kKeys, 1 << pool.page_shift);
        const bool copies = lane < 4 && (16 * lane & (rows - 1)) == 0;
        const auto look_up = [&](int i) {
            if (i >= n || lane >= 4) return -1;
            const int j = first_key(i) + 16 * lane;
            return j < len ? page_of(pool, s.index, j) : -1;
        };
        int page = -1, ahead = look_up(0), c = 0;
        for (; c < 2 * n; ++c) {
            const int slot = c % Sh::kSlots;
            if (!(c & 1)) {
                page = ahead;
                ahead = look_up(c / 2 + 1);
            }
            if (c >= Sh::kSlots && !guard.wait_all(raw_empty(slot), (c / Sh::kSlots - 1) & 1)) break;
            const unsigned there = __ballot_sync(0xffffffffu, page >= 0), from = __ballot_sync(0xffffffffu, page >= 0 && copies);
            if (lane == 0) {
                groups_there[slot] = there;
                mbar_expect_tx(raw_full(slot), __popc(from) * rows * (kRowBytes + (c & 1 ? 0 : 2 * G)));
            }
            __syncwarp();
            if (page >= 0 && copies) {
                const int64_t row = page_row(pool, page, hk, first_key(c / 2) + 16 * lane);
                const uint32_t to = ring_at + slot * Sh::kSlot;
                bulk_load(to + 16 * lane * kRowBytes, static_cast<const uint8_t*>(c & 1 ? pool.v : pool.k) + row * kRowBytes, rows * kRowBytes, raw_full(slot));
                if (!(c & 1)) {
                    bulk_load(to + Sh::kCodes + 16 * lane * G, pool.k_scale + row * G, rows * G, raw_full(slot));
                    bulk_load(to + Sh::kCodes + (kKeys + 16 * lane) * G, pool.v_scale + row * G, rows * G, raw_full(slot));
                }
            }
        }
        for (int i = max(0, c - Sh::kSlots); i < c; ++i) guard.settle(raw_full(i % Sh::kSlots), i / Sh::kSlots & 1);      // (whoever gave up, what is under way lands)
    } else if (warp >= Sh::kDecodes) {
        // ---- codes into fp16
        constexpr int kThreads = Sh::kDecoders * 32;
        const int dt = t - Sh::kDecodes * 32, side = dt >> 6, own_row = dt & 63;             // (scales: of the first 128)
        bool ok = true;
        const auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); };
        uint8_t* const stages = raw + (kv_at - smem_u32(raw));
        const auto one_piece = [&](uint8_t* stage, int u, Word w, uint32_t f, bool out) {
            uint32_t h[4];
            codes_f16(w, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = out ? 0u : times2(h[i], f);       // (0 times NaN is NaN)
            *reinterpret_cast<uint4*>(stage + swizzled(u / (4 * D32), u % (4 * D32), kKeys)) = make_uint4(h[0], h[1], h[2], h[3]);
        };
        const auto decode = [&](int c, bool masked, int j0, unsigned there) {
            uint8_t* const stage = stages + c % ST * Sh::kStage;
            const Word* const codes = reinterpret_cast<const Word*>(ring + c % Sh::kSlots * Sh::kSlot);
            const auto factor = [&](int u) { return factors[c & 1][u / (4 * D32)][kE2m1 ? u % (4 * D32) / 4 : 0]; };
            if (!masked && there == 0xFu) {
                Word w[P];
                uint32_t f[P];
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    w[k] = codes[dt + kThreads * k];
                    f[k] = factor(dt + kThreads * k);
                }
#pragma unroll
                for (int k = 0; k < P; ++k) one_piece(stage, dt + kThreads * k, w[k], f[k], false);
            } else {
#pragma unroll 1
                for (int u = dt; u < kThreads * P; u += kThreads) {
                    const int row = u / (4 * D32);
                    one_piece(stage, u, codes[u], factor(u), !(there >> (row >> 4) & 1u) || !(j0 + row < len && some_sees(lo, hi, j0 + row, a.window, a.n_sink)));
                }
            }
            __syncwarp();                                    // (the fence between these stores and the MMAs is the issuing thread's)
            if (lane == 0) {
                mbar_arrive(full(c % ST));
                mbar_arrive(raw_empty(c % Sh::kSlots));
            }
        };
        const auto room = [&](int c) { return c < ST || guard.wait_all(empty(c % ST), (c / ST - 1) & 1); };
        const auto codes_there = [&](int c) { return guard.wait_all(raw_full(c % Sh::kSlots), c / Sh::kSlots & 1); };
        for (int i = 0; i < n; ++i) {                        // (a warp that gave up goes on meeting the others)
            const int j0 = first_key(i);
            const bool masked = masks(j0);
            ok = ok && codes_there(2 * i);
            const unsigned there = groups_there[2 * i % Sh::kSlots];
            uint32_t scale[G], own = kScaleLeast + 127;
            if (dt < 128) {                                  // of one row, of keys or values (those that nobody sees may hold anything; without a page the least scale)
                const int j = j0 + own_row;
                const bool on = j < len && some_sees(lo, hi, j, a.window, a.n_sink), holds = on && (there >> (own_row >> 4) & 1u);
                const uint8_t* const b = ring + 2 * i % Sh::kSlots * Sh::kSlot + Sh::kCodes + dt * G;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    scale[g] = holds ? b[g] : 0u;
                    own = max(own, scale[g]);
                }
                const uint32_t top = __reduce_max_sync(0xffffffffu, own), low = __reduce_min_sync(0xffffffffu, on ? own : 255u);
                if (lane == 0) warp_top[warp - Sh::kDecodes] = make_uint2(top, low);
            }
            meet();                                          // (and nobody is with the last tile's factors any more)
            const int refs_here[2] = {static_cast<int>(max(warp_top[0].x, warp_top[1].x)), static_cast<int>(max(warp_top[2].x, warp_top[3].x))};
            const int least = static_cast<int>(min(warp_top[2].y, warp_top[3].y));
            const int far = (refs_here[1] - least > kSpread ? kFarValues : 0) | (refs_here[0] - static_cast<int>(min(warp_top[0].y, warp_top[1].y)) > kKeySpread<KIND> ? kFarKeys : 0);
            if (dt < 128) {
                const int ref = far & (side == 1 ? kFarValues : kFarKeys) ? static_cast<int>(own) : refs_here[side];
#pragma unroll
                for (int g = 0; g < G; ++g) factors[side][own_row][g] = power_f16(static_cast<int>(scale[g]) - ref + kCodeLift) * 0x10001u;
            }
            ok = ok && room(2 * i);                          // (the scales of kTileScales tiles ago have been read by then: stages hold three tiles at most, and the softmax is one behind)
            if (ok && dt < 128) {
                TileScales& to = scales[i % kTileScales];
                if (dt == 0) {
                    to.most_key = refs_here[0] - 127;
                    to.most = static_cast<float>(refs_here[1] - 127 - kCodeLift);
                    to.least = static_cast<float>(least - 127 - kCodeLift);
                    to.far = far;
                }
                if (side == 1) to.exponent[own_row] = static_cast<float>(static_cast<int>(own) - 127 - kCodeLift);
                else to.key[own_row] = static_cast<int>(own) - 127;
            }
            meet();
            if (ok) decode(2 * i, masked, j0, there);
            ok = ok && codes_there(2 * i + 1) && room(2 * i + 1);
            if (ok) decode(2 * i + 1, masked, j0, there);
        }
    } else if (warp == Sh::kIssues && n > 0) {
        const uint32_t idesc_s = idesc_16<true>(kKeys), idesc_o = idesc_16<true>(D) | kRowsAreContraction;
        const bool one = elect_one();
        const auto fence = [] { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); };
        const auto scores = [&](int i) {                     // S of tile i; its keys' stage is free when it is there
            const int st = 2 * i % ST;
#pragma unroll
            for (int w = 0; w < T; ++w) {
#pragma unroll
                for (int b = 0; b < Sh::kDB; ++b)
                    umma_box(2, tmem + w * Sh::kOf + (i & 1) * kKeys, smem_desc_sw128(q_at + (w * Sh::kDB + b) * kRows * 128), smem_desc_sw128(kv_at + st * Sh::kStage + b * kKeys * 128), idesc_s,
                             min(4, D / 16 - 4 * b), b > 0);
                umma_commit(s_full(w, i & 1));
            }
            umma_commit(empty(st));
        };
        bool ok = guard.wait_all(q_full, 0) && guard.wait_all(full(0), 0);
        if (ok && one) {
            fence();
            tc_fence_after();
            scores(0);
        }
        __syncwarp();
        for (int i = 0; i < n && ok; ++i) {
            if (i + 1 < n) {
                ok = guard.wait_all(full((2 * i + 2) % ST), (2 * i + 2) / ST & 1);
                if (ok && one) {
                    fence();
                    tc_fence_after();
                    scores(i + 1);
                }
                __syncwarp();
            }
            const int c = 2 * i + 1, st = c % ST;
            ok = ok && guard.wait_all(full(st), c / ST & 1);
            for (int w = 0; w < T && ok; ++w) {
                ok = guard.wait_all(p_full(w, i & 1), i / 2 & 1);
                if (ok && one) {
                    fence();
                    tc_fence_after();
                    for (int k = 0; k < kKeys / 16; ++k)
                        umma_bf16_ts(tmem + w * Sh::kOf + Sh::kO, tmem + w * Sh::kOf + (i & 1) * kKeys + 8 * k, smem_desc_rows_sw128(kv_at + st * Sh::kStage + k * 2048, kKeys * 128), idesc_o,
                                     i > 0 || k > 0);
                    umma_commit(o_step(w));
                }
                __syncwarp();
            }
            if (ok && one) umma_commit(empty(st));
            __syncwarp();
        }
        if (one) umma_commit(ok ? o_full : ended);
        __syncwarp();
        guard.settle(ok ? o_full : ended, 0);                // (whoever else gave up, the tensor memory is not given back under an MMA)
    } else if (warp < 4 * T) {
        // ---- softmax, a thread per row
        const int w = warp >> 2, r = t & (kRows - 1), i_row = q0 + w * per + r / a.pack, head = head0 + r % a.pack;
        const bool mine = r < per * a.pack && i_row < s.n_q;
        const int p = mine ? query_pos(a, s, len, i_row) : -1;
        // of a score: fraction 2^(key - lifted) for the exponent of its key's scale
        const float fraction = __uint_as_float((__float_as_uint(a.scale_log2) & 0x7FFFFFu) | 0x3F800000u);
        int lifted = kCodeLift - (static_cast<int>(__float_as_uint(a.scale_log2) >> 23) - 127);
        if (n > 0) {                                         // this row's queries, in fp16
            const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(a.q) + ((s.q_row + i_row) * a.n_heads + head) * D;
            uint32_t top = 0;
            if (mine) {
#pragma unroll
                for (int c = 0; c < D; c += 8) {
                    const uint4 y = *reinterpret_cast<const uint4*>(q + c);
                    constexpr uint32_t some = 0x7FFF7FFFu;
                    top = __vmaxu2(top, __vmaxu2(__vmaxu2(y.x & some, y.y & some), __vmaxu2(y.z & some, y.w & some)));
                }
            }
            top = max(top & 0xFFFFu, top >> 16);
            const int e = top ? min(max(14 - (static_cast<int>(top >> 7) - 127), -113), 126) : 0;      // (2^126 times the smallest ones at most)
            const float lift = two_to(e);
            lifted += e;
#pragma unroll 4
            for (int c = 0; c < D; c += 8) {
                uint4 y = make_uint4(0, 0, 0, 0);
                if (mine) y = *reinterpret_cast<const uint4*>(q + c);
                uint32_t x[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = two_f16(__uint_as_float(x[i] << 16) * lift, __uint_as_float(x[i] & 0xFFFF0000u) * lift);
                store16(q_at + w * (Sh::kDB * kRows * 128) + swizzled(r, c / 8, kRows), x);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
        }
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;        // this warp's 32 lanes
        const uint32_t o_col = tmem + w * Sh::kOf + Sh::kO + lanes;
        // Reference of the scores (in powers of two), what that of weights times scales lies above it, sum of the weights (against the first, less kF16Lift); O: against the second, likewise.  (The second is
        // no number of its own: beside a score of 2^17 the exponents of scales lose their last bits.)
        float m = -CUDART_INF_F, above = -CUDART_INF_F, l = 0.f;
        bool masked = false;
        uint32_t visible[kKeys / 32];                        // a bit for every key of the tile that the row sees
        const auto look = [&](int i) {
            const int j0 = first_key(i);
            masked = masks(j0);
            if (!masked) return;
            const int past = min(p, len - 1) - j0 + 1, from = max(p - a.window + 1, 0) - j0, sink = a.n_sink - j0;
#pragma unroll
            for (int x = 0; x < kKeys / 32; ++x) visible[x] = below(past - 32 * x) & (~below(from - 32 * x) | below(sink - 32 * x));
        };
        const auto scores_there = [&](int i) { return guard.wait_all(s_full(w, i & 1), i / 2 & 1); };
        const auto weigh = [&](int i) {
            const int buf = i & 1;
            tc_fence_after();
            const TileScales& of = scales[i % kTileScales];
            const uint32_t s_col = tmem + w * Sh::kOf + buf * kKeys + lanes;
            float scale = score_scale(fraction, of.most_key, lifted);
            if (of.far & kFarKeys) {
                scale_scores(s_col, of.key, fraction, lifted);
                scale = 1.f;
            }
            const uint32_t sees0 = masked ? visible[0] : 0xFFFFFFFFu, sees1 = masked ? visible[1] : 0xFFFFFFFFu;
            const uint64_t scale2 = two_f32(scale, scale);
            const auto scores_of = [&](int c0, float (&x)[32]) {
                tmem_ld_cols<32>(s_col + c0, x);
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) x[c] = visible[c0 / 32] >> c & 1u ? x[c] : -CUDART_INF_F;
                }
            };
            float tops[4];
            {
                float x[kKeys];
                tmem_ld_cols<kKeys>(s_col, x);
                if (masked) {
#pragma unroll
                    for (int c = 0; c < kKeys; ++c) x[c] = visible[c / 32] >> (c & 31) & 1u ? x[c] : -CUDART_INF_F;
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) tops[b] = x[b];
#pragma unroll
                for (int c = 4; c < kKeys; c += 8) {         // (three at a time)
#pragma unroll
                    for (int b = 0; b < 4; ++b) tops[b] = c + 4 + b < kKeys ? fmaxf(fmaxf(tops[b], x[c + b]), x[c + 4 + b]) : fmaxf(tops[b], x[c + b]);
                }
            }
            const float top = __fmul_rn(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), scale);      // (scale is positive; rounded before anything is taken from it)
            if (top - m > kMoveAt) {
                const float up = top - m;                    // (infinite where there was nothing yet)
                l *= ex2_approx(-up);
                above -= up;
                m = top;
            }
            const bool some = m > -CUDART_INF_F, far = (of.far & kFarValues) != 0 || __any_sync(0xffffffffu, some && fabsf(m) > kLargeScore);
            const float ref = some ? m : 0.f, here = top - ref;
            if (__any_sync(0xffffffffu, here + of.most > above + kMoveAt)) {
                const float top_w = of.far & kFarValues ? top_product(s_col, sees0, sees1, of.exponent, scale, ref) : here + of.least;
                const bool move = top_w > above + kMoveScaledAt;
                if (i > 0 && __any_sync(0xffffffffu, move)) {
                    // (the step before may still be adding; the one before that was complete before this S was)
                    if (!guard.wait_all(o_step(w), (i - 1) & 1)) return false;
                    tc_fence_after();
                    const float f = move ? ex2_approx(above - top_w) : 1.f;
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        uint32_t y[32];
                        tmem_ld_cols<32>(o_col + c, o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) y[k] = __float_as_uint(o[k] * f);
                        tmem_st_cols<32>(o_col + c, y);
                    }
                }
                if (move) above = top_w;
            }
            // The weights as they meet the values are those that have the sum, in other units, as long as a tile's values have one scale (2^64 above the scores' reference nothing is left of the
            // tile's values, and the units may be smaller).
            const float off = far || !some ? 0.f : fminf(above - of.most, 64.f);
            const uint64_t ref2 = two_f32(kF16Lift - (ref + off), kF16Lift - (ref + off));
            uint64_t sums[2] = {0, 0};
            if (!far) {
#pragma unroll
                for (int c0 = 0; c0 < kKeys; c0 += 32) {
                    float x[32];
                    uint32_t weights[16];
                    scores_of(c0, x);
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        float y, z;
                        split_f32(fma_f32x2(two_f32(x[c], x[c + 1]), scale2, ref2), y, z);
                        y = ex2_approx(y);
                        z = ex2_approx(z);
                        sums[c / 2 & 1] = add_f32x2(sums[c / 2 & 1], two_f32(y, z));
                        weights[c / 2] = two_f16(y, z);      // (rounded for the product alone)
                    }
                    tmem_st_cols<16>(s_col + c0 / 2, weights);
                }
            } else {
                sums[0] = two_f32(weigh_far(s_col, sees0, sees1, of.far & kFarValues ? of.exponent : nullptr, of.most, scale, ref, some ? above : 0.f), 0.f);
            }
            float even, odd;
            split_f32(add_f32x2(sums[0], sums[1]), even, odd);
            l = fmaf(even + odd, ex2_approx(off), l);
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(p_full(w, buf));
            return true;
        };
        bool ok = walk_tiles(0, n, 1, look, scores_there, weigh);
        // ---- the rows
        if (ok && n > 0) ok = guard.wait_all(o_full, 0);
        tc_fence_after();
        const int64_t part = s.part0 + static_cast<int64_t>(part_of_seq) * s.n_q + i_row;
        float4* const sums = reinterpret_cast<float4*>(raw + (q_at - smem_u32(raw)));         // of a cluster's CTA (sums_at)
        // (by halves: of values near 2^-117 the factor is no normal number)
        const float half = l > 0.f ? exp2f(0.5f * above) : 0.f, by = half * (s.parts > 1 || ranks > 1 || !(l > 0.f) ? 1.f : 1.f / l);
        m -= kF16Lift;
        for (int c = 0; c < D && ok; c += 32) {
            float o[32];
            if (n > 0) tmem_ld_cols<32>(o_col + c, o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = l > 0.f ? o[k] * half * by : 0.f;
            if (ranks > 1) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) sums[sums_at(w * kRows + r, (c + k) / 4, D)] = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                continue;
            }
            if (!mine) continue;
            if (s.parts > 1) {
                float* const dst = a.part_o + (part * a.n_heads + head) * D + c;
#pragma unroll
                for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            } else {
                __nv_bfloat16* const dst = static_cast<__nv_bfloat16*>(a.out) + ((s.q_row + i_row) * a.n_heads + head) * D + c;
#pragma unroll
                for (int k = 0; k < 32; k += 8) store8(dst + k, o + k);
            }
        }
        if (ranks > 1) row_ml[w][r] = make_float2(m, l);
        if (mine && ok && ranks == 1) {
            if (s.parts > 1) a.part_ml[part * a.n_heads + head] = make_float2(m, l);
            else if (a.lse) a.lse[(s.q_row + i_row) * a.n_heads + head] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;      // ln 2
        }
        tc_fence_before();
    }
    __syncthreads();
    // (before the cluster meets: who holds tensor memory waits for no other CTA, which may wait for some of it behind another launch's)
    if (warp == Sh::kIssues) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::kColumns);
    }
    if (ranks > 1) {                                         // (reached by all CTAs of the cluster, whoever gave up)
        cluster_arrive_release();
        cluster_wait_acquire();
        join_cluster<T>(a, s, q_at, smem_u32(row_ml), reinterpret_cast<float*>(raw + (q_at - smem_u32(raw)) + T * D * kRows * 4), ranks, q0, per, head0, part_of_seq);
        cluster_arrive_release();                            // (nobody's sums are gone while another reads them)
        cluster_wait_acquire();
    }
}

template <int KIND, int D32, int T>
cudaError_t attend(const AttArgs& a, const PagePool& pool, cudaStream_t stream)
{
    static KernelSetup setup;
    using Sh = PageTileShape<KIND, D32, T>;
    const size_t smem = smem_for_tmem(Sh::kSmem, Sh::kColumns);              // (no CTA more than there is tensor memory for)
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(page_tile_kernel<KIND, D32, T>), smem, Sh::kColumns);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_blocks) * static_cast<unsigned>(a.n_heads / a.pack) * static_cast<unsigned>(a.cluster));
    cfg.blockDim = dim3(Sh::kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(a.cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, page_tile_kernel<KIND, D32, T>, a, pool);
}
template <int KIND, int D32>
cudaError_t by_tiles(int row_tiles, const AttArgs& a, const PagePool& pool, cudaStream_t stream)
{
    if constexpr (D32 <= 4)                                  // (two tiles of rows of larger heads have no room in tensor memory)
        if (row_tiles == 2) return attend<KIND, D32, 2>(a, pool, stream);
    return attend<KIND, D32, 1>(a, pool, stream);
}
template <int KIND>
cudaError_t by_dim(int row_tiles, const AttArgs& a, const PagePool& pool, cudaStream_t stream)
{
    switch (a.head_dim / 32) {
    case 2: return by_tiles<KIND, 2>(row_tiles, a, pool, stream);
    case 3: return by_tiles<KIND, 3>(row_tiles, a, pool, stream);
    case 4: return by_tiles<KIND, 4>(row_tiles, a, pool, stream);
    case 5: return by_tiles<KIND, 5>(row_tiles, a, pool, stream);
    case 6: return by_tiles<KIND, 6>(row_tiles, a, pool, stream);
    case 7: return by_tiles<KIND, 7>(row_tiles, a, pool, stream);
    default: return by_tiles<KIND, 8>(row_tiles, a, pool, stream);
    }
}

}  // namespace

cudaError_t launch_page_decode(int kind, int row_tiles, const AttArgs& a, const PagePool& pool, cudaStream_t stream)
{
    return kind == MVLA_PAGE_E4M3 ? by_dim<MVLA_PAGE_E4M3>(row_tiles, a, pool, stream) : by_dim<MVLA_PAGE_E2M1>(row_tiles, a, pool, stream);
}

}  // namespace mvla
