// Attention of single tokens over a cache in pages: at most 16 query rows of a sequence share a key head.  e4m3 or e2m1, and for small heads and short sequences the rows' own type
// (bf16).
//
// Bound by the bytes of the pages, and by unpacking them.  A warp takes tiles of 16 or 32 keys as the registers that the tensor cores read (m16n8k16):
// keys are the 16 rows of the first product, columns of the values those of the second, query rows the 8 columns of both.  Which element of the
// head meets which is free as long as queries and keys agree, so a lane copies runs of its own, a tile ahead, asynchronously, and no lane waits for
// another's but for the scales, which all of them read.  16 rows of a tile never cross a page, so that a page number is looked up once for 16 keys, a tile before its copies begin.
//   Quantised keys and values become fp16 in registers, which holds every code; values of two keys are interleaved before that, in their 8 or 4 bits,
// which makes them the second product's operand.  Scales are powers of two.  One a row (e4m3): a key's multiplies its scores; a value's is added to
// the exponent of its weight, w = 2^((x - reference) + (e - above)).  So there are two references and two exponentials: those of the weights that meet the values, `above` the other, and those
// of the sum that divides them.  (Scores are taken from their reference first: beside a score of 2^17 the exponents of scales lose their last bits.)  One for 32 elements (e2m1): the row's largest is taken as above, the rest of it multiplies the codes (2^13 times
// the quotient of the scales: 6 2^13 is a number of fp16, and a group 2^-27 of the largest one is nothing).  Queries are fp16 too, every row
// times a power of two that puts its largest element between 2^14 and 2^15.  bf16 weights (unquantised pages) meet the values in two
// parts, what the type holds and what it leaves; fp16 ones are one part, in units of 2^-kF16Lift of their reference.
//   A sequence's visible keys are cut into parts of about the same length over the whole batch; a CTA is four warps that take the part's tiles in turn.  The
// parts of a cluster are joined through its shared memory, and clusters (where a sequence has more than one) by a kernel behind.
//
// B200, 32 query heads over 8 heads of 128, with the join: 16 tokens over 500 to 4000 e4m3 rows 27 us (75 MB; launch, the first copies and the end of a CTA 9, the join 4,
// 5 TB/s in between); one token over 131072 rows of e4m3 64 us (4.2 TB/s), of e2m1 53 us: 64 conversions of two codes and as many products of pairs to 16 keys, of
// the instructions' pipe 47 %, latency beside them (16 warps to a multiprocessor).  Tiles of 32 keys with one ahead: 53 us, of 16 keys 55, two ahead 56 (three CTAs fit instead of four).
#include "attend_tile.cuh"
#include "page.cuh"

#include <cfloat>

namespace mvla {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = kPageTokenStages;
constexpr float kNothing = -FLT_MAX;         // reference of a row that has seen nothing yet

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int there)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t bits_of(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat162 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ uint32_t times(uint32_t x, uint32_t f)
{
    return bits_of(__hmul2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&f)));
}
// The transpose of an 8 x 8 block of 16-bit values, a pair of neighbours in every lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight codes as they lie in memory, and how many runs of eight a lane copies at once at most: of a key's row, of a value's.
template <int KIND> struct Run;
template <> struct Run<MVLA_PAGE_ROWS> { using Word = uint4; static constexpr int kKeyRuns = 1, kValueRuns = 1; };
template <> struct Run<MVLA_PAGE_E4M3> { using Word = uint2; static constexpr int kKeyRuns = 2, kValueRuns = 2; };
template <> struct Run<MVLA_PAGE_E2M1> { using Word = uint32_t; static constexpr int kKeyRuns = 4, kValueRuns = 2; };

// A warp's tile in shared memory: every lane's runs of its rows of keys (g, g + 8 of 16), of values (2 c, 2 c + 1, 2 c + 8, 2 c + 9), and the scales of keys
// and values.  Runs of a key's row: D32, four lanes side by side; in lots of kKeyRuns, then halves of those, that one lane has next to one another.  Runs of
// a value's row: M64, eight lanes side by side, likewise.
template <int KIND, int D32>
struct Tile {
    static constexpr int kM64 = (D32 + 1) / 2, kSub = page_token_sub(KIND, D32), kKeys = 16 * kSub;
    static constexpr int kRun = static_cast<int>(sizeof(typename Run<KIND>::Word));
    static constexpr int kKeyRow = D32 * 32 * kRun, kValueRow = kM64 * 32 * kRun;       // of a lane's row, for the whole warp
    static constexpr int kGroups = page_row_scales(KIND, D32 * 32);
    static constexpr int kRows = kSub * (2 * kKeyRow + 4 * kValueRow), kScales = kSub * 2 * 16 * kGroups;
    static constexpr int kBytes = kRows + kScales;
    static_assert(kBytes == page_token_tile(KIND, D32), "the plan's size");
    // runs i .. i + n - 1 of a lane lie together: how many, and the first
    static __device__ __forceinline__ constexpr int lot(int i, int all, int most)
    {
        int n = most;
        while (i / n * n + n > all) n /= 2;
        return n;
    }
    // first element of run i of lane c's keys, first column of run m of lane g's values
    static __device__ __forceinline__ constexpr int element(int i, int c)
    {
        const int n = lot(i, D32, Run<KIND>::kKeyRuns);
        return i / n * n * 32 + 8 * n * c + 8 * (i % n);
    }
    static __device__ __forceinline__ constexpr int column(int m, int g)
    {
        const int n = lot(m, D32 / 2, Run<KIND>::kValueRuns);
        return m < D32 / 2 ? m / n * n * 64 + 8 * n * g + 8 * (m % n) : 64 * m + 8 * g;
    }
    // where run i of a lane lies in its row of the tile
    static __device__ __forceinline__ constexpr int key_at(int i, int lane)
    {
        const int n = lot(i, D32, Run<KIND>::kKeyRuns);
        return (i / n * n * 32 + lane * n + i % n) * kRun;
    }
    static __device__ __forceinline__ constexpr int value_at(int m, int lane)
    {
        const int n = m < D32 / 2 ? lot(m, D32 / 2, Run<KIND>::kValueRuns) : 1;
        return (m / n * n * 32 + lane * n + m % n) * kRun;
    }
};

// N runs that lie next to one another (16 bytes at most).
template <int N, class W>
__device__ __forceinline__ void load_runs(const uint8_t* p, W* w)
{
    if constexpr (N * sizeof(W) == 16) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        memcpy(w, &x, 16);
    } else if constexpr (N * sizeof(W) == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        memcpy(w, &x, 8);
    } else {
        static_assert(N == 1, "runs");
        w[0] = *reinterpret_cast<const W*>(p);
    }
}
// The number that eight bits stand for, less `off`, without the conversion's pipe.
__device__ __forceinline__ float byte_float(uint32_t byte, int off) { return __uint_as_float(0x4B000000u + byte) - static_cast<float>(8388608 + off); }

template <int KIND, int D32, int NR>
__global__ void __launch_bounds__(kWarps * 32, page_token_ctas(KIND, D32, NR)) page_token_kernel(const __grid_constant__ AttArgs a, const __grid_constant__ PagePool pool)
{
    using Sh = Tile<KIND, D32>;
    using Word = typename Run<KIND>::Word;
    constexpr bool kScaled = KIND != MVLA_PAGE_ROWS, kE2m1 = KIND == MVLA_PAGE_E2M1;
    constexpr int D = D32 * 32, M64 = Sh::kM64, U = Sh::kSub, G = Sh::kGroups;
    constexpr float kLift = kScaled ? kF16Lift : 0.f;
    constexpr int kCodeLift = kE2m1 ? 13 : 0;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint4 q_frag[D32][NR][32];
    __shared__ float merge_m[kWarps][16], merge_f[kWarps][16], merge_l[kWarps][16];
    __shared__ float2 cta_ml[16], peer_ml[kMaxCluster][8 * NR];
    __shared__ float q_lift[16], q_scale[16], q_half[16];    // what a row's queries are multiplied by; what that makes of the scores' scale, in two factors of about the same size
    __shared__ __align__(4) uint16_t factors[kE2m1 ? kWarps : 1][kE2m1 ? U : 1][2][kE2m1 ? D32 : 1][16];      // of the groups of a tile's rows, fp16
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, g = lane >> 2, c = lane & 3;
    const AttSeq& s = a.s[seq_of_block(a, blockIdx.x)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads, n_rows = s.n_q * group, len = seq_len(a, s);
    int p[NR][2];                                            // positions of this lane's rows 8 n + 2 c + e
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * c + e;
            p[n][e] = r < n_rows ? query_pos(a, s, len, r / group) : -1;
        }
    const int lo = query_pos(a, s, len, 0), hi = query_pos(a, s, len, s.n_q - 1);
    const TileRange range = tile_range(a, len, lo, hi, Sh::kKeys);
    // (s.parts: clusters; each CTA of one takes a part)
    const int ranks = cluster_ctas(), rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int part = static_cast<int>(blockIdx.x) - s.blk0, parts = s.parts * ranks, per_part = (range.count + parts - 1) / parts;
    const int t0 = part * per_part, t1 = min(range.count, t0 + per_part);
    // o[m][i][n]: columns column(m, g) + 2 i and + 1 (values 0, 1 and 2, 3), rows 8 n + 2 c and + 1
    float o[M64][4][NR][4];
#pragma unroll
    for (int m = 0; m < M64; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NR; ++n) o[m][i][n][0] = o[m][i][n][1] = o[m][i][n][2] = o[m][i][n][3] = 0.f;
    // reference of the sum, what that of the weights as they meet the values lies above it (nothing where there are no scales), the sum
    float ref[NR][2], above[NR][2], sum[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { ref[n][e] = kNothing; above[n][e] = sum[n][e] = 0.f; }

    // Tile t0 + warp + kWarps u is this warp's u-th.  Page of its keys 16 (lane / 16) ... (of the first sixteen, where a tile has no more):
    const int mine = t1 > t0 + warp ? (t1 - t0 - warp + kWarps - 1) / kWarps : 0;
    const auto first_key = [&](int u) { return range.tile(t0 + warp + kWarps * u) * Sh::kKeys; };
    const auto look_up = [&](int u) {
        if (u >= mine) return -1;
        const int j = first_key(u) + (U > 1 ? lane & 16 : 0);
        return j < len ? page_of(pool, s.index, j) : -1;
    };
    uint8_t* const stages = ring + warp * kStages * Sh::kBytes;
    const uint32_t stages_at = smem_u32(stages);
    const int row_bytes = page_row_bytes(KIND, D, 2);
    const uint8_t* const kb = static_cast<const uint8_t*>(pool.k);
    const uint8_t* const vb = static_cast<const uint8_t*>(pool.v);
    // starts the copies of a tile (always a group of copies, an empty one too)
    const auto fetch = [&](int u, int stage, int page) {
        if (u < mine) {
            const int j0 = first_key(u);
            uint32_t dst = stages_at + stage * Sh::kBytes;
#pragma unroll
            for (int v = 0; v < U; ++v, dst += 2 * Sh::kKeyRow + 4 * Sh::kValueRow) {
                const int pg = __shfl_sync(0xffffffffu, page, 16 * v);
                const bool there = pg >= 0;
                const int64_t row0 = there ? page_row(pool, pg, hk, j0 + 16 * v) : 0;
                const uint8_t* const k0 = kb + row0 * row_bytes;
                const uint8_t* const v0 = vb + row0 * row_bytes;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < D32; ++i) {
                        constexpr int most = Run<KIND>::kKeyRuns;
                        const int lot = Sh::lot(i, D32, most);
                        if (i % lot) continue;
                        const uint32_t to = dst + n * Sh::kKeyRow + Sh::key_at(i, lane);
                        const uint8_t* const from = k0 + (g + 8 * n) * row_bytes + Sh::element(i, c) / 8 * Sh::kRun;
                        if (lot == 4) copy_async<(4 * Sh::kRun > 16 ? 16 : 4 * Sh::kRun)>(to, from, there);
                        else if (lot == 2) copy_async<(2 * Sh::kRun > 16 ? 16 : 2 * Sh::kRun)>(to, from, there);
                        else copy_async<Sh::kRun>(to, from, there);
                    }
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int m = 0; m < M64; ++m) {
                        const int lot = m < D32 / 2 ? Sh::lot(m, D32 / 2, Run<KIND>::kValueRuns) : 1;
                        if (m % lot) continue;
                        if (m >= D32 / 2 && g >= 4) continue;
                        const uint32_t to = dst + 2 * Sh::kKeyRow + n * Sh::kValueRow + Sh::value_at(m, lane);
                        const uint8_t* const from = v0 + (2 * c + (n & 1) + 8 * (n >> 1)) * row_bytes + Sh::column(m, g) / 8 * Sh::kRun;
                        if (lot == 2) copy_async<(2 * Sh::kRun > 16 ? 16 : 2 * Sh::kRun)>(to, from, there);
                        else copy_async<Sh::kRun>(to, from, there);
                    }
                if constexpr (kScaled) {                     // (16 rows' scales lie side by side: 16 bytes a lane)
                    if (lane < 2 * G) {
                        const uint8_t* const from = (lane < G ? pool.k_scale : pool.v_scale) + row0 * G + lane % G * 16;
                        copy_async<16>(stages_at + stage * Sh::kBytes + Sh::kRows + (v * 2 * G + lane) * 16, from, there);
                    }
                }
            }
        }
        copies_done();
    };
    int ahead[kStages - 1];
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) ahead[u] = look_up(u);
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u, u, ahead[u]);
    int next = look_up(kStages - 1);
    // ---- queries: the first product's operand
    const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(a.q);
    const auto query = [&](int r) { return q + ((s.q_row + r / group) * a.n_heads + hk * group + r % group) * D; };
    for (int r = warp; r < 8 * NR; r += kWarps) {
        uint32_t top = 0;
        if (kScaled && r < n_rows)
            for (int i = 2 * lane; i < D; i += 64) top = __vmaxu2(top, *reinterpret_cast<const uint32_t*>(query(r) + i) & 0x7FFF7FFFu);
        top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
        if (lane == 0) {
            const int e = kScaled && top ? max(14 - (static_cast<int>(top >> 7) - 127), -113) : 0;       // (2^126 times the smallest ones at most)
            // (with their product, or with a key's scale in one step, the scale could leave the normal numbers though the scores do not)
            const uint32_t bits = __float_as_uint(a.scale_log2);
            const int power = static_cast<int>(bits >> 23) - 127 - min(e, 126), half = kScaled ? power >> 1 : 0;
            q_lift[r] = two_to(min(e, 126));
            q_scale[r] = __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u) * two_to(power - half);
            q_half[r] = two_to(half);
        }
    }
    __syncthreads();
    for (int u = t; u < D32 * NR * 32; u += kWarps * 32) {
        const int piece = u / (NR * 32), n = u / 32 % NR, l = u & 31, r = (l >> 2) + 8 * n;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (r < n_rows) w = *reinterpret_cast<const uint4*>(query(r) + Sh::element(piece, l & 3));
        if constexpr (kScaled) {
            const float f = q_lift[r];
            uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = bits_of(__floats2half2_rn(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xFFFF0000u) * f));
            w = make_uint4(x[0], x[1], x[2], x[3]);
        }
        q_frag[piece][n][l] = w;
    }
    __syncthreads();
    float q_by[NR][2], q_key[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { q_by[n][e] = q_scale[8 * n + 2 * c + e]; q_key[n][e] = q_half[8 * n + 2 * c + e]; }

    int stage = 0;
    for (int u = 0; u < mine; ++u, stage = stage + 1 < kStages ? stage + 1 : 0) {
        const int then = look_up(u + kStages);
        wait_copies<kStages - 2>();
        __syncwarp();                                        // (every lane's copies are there; nobody reads the last tile any more)
        fetch(u + kStages - 1, stage > 0 ? stage - 1 : kStages - 1, next);
        next = then;
        const int j0 = first_key(u);
        const bool all = j0 + Sh::kKeys - 1 <= lo && (hi - j0 < a.window || j0 + Sh::kKeys - 1 < a.n_sink);      // (lo is below the length)
        const uint8_t* const tile = stages + stage * Sh::kBytes;
        int largest[U];                                      // e2m1: byte of the largest scale of key lane % 16, or of its values (lanes 16 ...)
        if constexpr (kE2m1) {
#pragma unroll
            for (int v = 0; v < U; ++v) {
                const uint8_t* const bytes = tile + Sh::kRows + v * 2 * G * 16 + lane * G;
                int b[D32], top = 0;
                if constexpr (D32 % 4 == 0) {
#pragma unroll
                    for (int i = 0; i < D32; i += 4) {
                        const uint32_t w = *reinterpret_cast<const uint32_t*>(bytes + i);
#pragma unroll
                        for (int k = 0; k < 4; ++k) b[i + k] = w >> (8 * k) & 0xFFu;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < D32; ++i) b[i] = bytes[i];
                }
#pragma unroll
                for (int i = 0; i < D32; ++i) top = max(top, b[i]);
                largest[v] = top;
                // 2^(13 + difference) in fp16, nothing below its normal numbers
#pragma unroll
                for (int i = 0; i < D32; ++i) factors[warp][v][lane >> 4][i][lane & 15] = static_cast<uint16_t>(max(b[i] - top + 15 + kCodeLift, 0) << 10);
            }
            __syncwarp();
        }
        // x[v][n][2 k + e]: key 16 v + g + 8 k, row 8 n + 2 c + e
        float x[U][NR][4] = {};
#pragma unroll
        for (int i0 = 0; i0 < D32; ++i0) {
            const int lot = Sh::lot(i0, D32, Run<KIND>::kKeyRuns);
            if (i0 % lot) continue;
            uint4 y[4][NR];
#pragma unroll
            for (int i = 0; i < lot; ++i)
#pragma unroll
                for (int n = 0; n < NR; ++n) y[i][n] = q_frag[i0 + i][n][lane];
#pragma unroll
            for (int v = 0; v < U; ++v) {
                const uint8_t* const rows = tile + v * (2 * Sh::kKeyRow + 4 * Sh::kValueRow) + Sh::key_at(i0, lane);
                Word k0[4], k1[4];
                if (lot == 4 && kE2m1) {
                    load_runs<kE2m1 ? 4 : 1>(rows, k0);
                    load_runs<kE2m1 ? 4 : 1>(rows + Sh::kKeyRow, k1);
                } else if (lot == 2 && kScaled) {
                    load_runs<kScaled ? 2 : 1>(rows, k0);
                    load_runs<kScaled ? 2 : 1>(rows + Sh::kKeyRow, k1);
                } else {
                    load_runs<1>(rows, k0);
                    load_runs<1>(rows + Sh::kKeyRow, k1);
                }
                uint32_t f0 = 0, f1 = 0;
                if constexpr (kE2m1) {
                    const int gr = i0 + (lot == 4 ? c : lot == 2 ? c >> 1 : 0);
                    f0 = factors[warp][v][0][gr][g] * 0x10001u;
                    f1 = factors[warp][v][0][gr][g + 8] * 0x10001u;
                }
#pragma unroll
                for (int i = 0; i < lot; ++i) {
                    uint32_t w0[4], w1[4];
                    if constexpr (KIND == MVLA_PAGE_ROWS) {
                        w0[0] = k0[i].x; w0[1] = k0[i].y; w0[2] = k0[i].z; w0[3] = k0[i].w;
                        w1[0] = k1[i].x; w1[1] = k1[i].y; w1[2] = k1[i].z; w1[3] = k1[i].w;
                    } else if constexpr (KIND == MVLA_PAGE_E4M3) {
                        from_e4m3(k0[i].x, w0[0], w0[1]);
                        from_e4m3(k0[i].y, w0[2], w0[3]);
                        from_e4m3(k1[i].x, w1[0], w1[1]);
                        from_e4m3(k1[i].y, w1[2], w1[3]);
                    } else {
                        from_e2m1(k0[i], w0);
                        from_e2m1(k1[i], w1);
#pragma unroll
                        for (int h = 0; h < 4; ++h) { w0[h] = times(w0[h], f0); w1[h] = times(w1[h], f1); }
                    }
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        mma16<kScaled>(x[v][n], w0[0], w1[0], w0[1], w1[1], y[i][n].x, y[i][n].y);
                        mma16<kScaled>(x[v][n], w0[2], w1[2], w0[3], w1[3], y[i][n].z, y[i][n].w);
                    }
                }
            }
        }
        float of_value[U][2];                                // exponent of the scale of key g + 8 k's values
#pragma unroll
        for (int v = 0; v < U; ++v) {
            uint32_t kbyte[2] = {127, 127};
            of_value[v][0] = of_value[v][1] = 0.f;
            if constexpr (KIND == MVLA_PAGE_E4M3) {
                const uint8_t* const bytes = tile + Sh::kRows + v * 32;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    kbyte[k] = bytes[g + 8 * k];
                    of_value[v][k] = byte_float(bytes[16 + g + 8 * k], 127);
                }
            } else if constexpr (kE2m1) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    kbyte[k] = static_cast<uint32_t>(__shfl_sync(0xffffffffu, largest[v], g + 8 * k));
                    of_value[v][k] = byte_float(static_cast<uint32_t>(__shfl_sync(0xffffffffu, largest[v], 16 + g + 8 * k)), 127 + kCodeLift);
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float by = __uint_as_float(kbyte[k] ? kbyte[k] << 23 : 0x400000u) * (kE2m1 ? 0x1p-13f : 1.f);      // (without the codes' lift; the least byte is 2^-127)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // (rounded before anything is taken from it; a score of nothing stays nothing)
                        float& y = x[v][n][2 * k + e];
                        y = __fmul_rn(y, q_by[n][e]);
                        if (kScaled) y = __fmul_rn(y, fminf(by * q_key[n][e], FLT_MAX));
                    }
                }
        }
        uint32_t seen[U][2] = {};                            // four bits for every key g + 8 k: which lanes have a row that sees it
        if (!all) {
#pragma unroll
            for (int v = 0; v < U; ++v)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int j = j0 + 16 * v + g + 8 * k, at = j < len ? j : -1;
                    bool some = false;
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const bool on = sees(p[n][e], at, a.window, a.n_sink);
                            some |= on;
                            if (!on) x[v][n][2 * k + e] = -CUDART_INF_F;
                        }
                    seen[v][k] = __ballot_sync(0xffffffffu, some);
                }
        }
        // references
        float top[NR][2];
        bool move = false;
        const auto top_product = [&](int n, int e) {         // from the reference on
            float w = fmaxf((x[0][n][e] - ref[n][e]) + of_value[0][0], (x[0][n][2 + e] - ref[n][e]) + of_value[0][1]);
            if (U > 1) w = fmaxf(w, fmaxf((x[U - 1][n][e] - ref[n][e]) + of_value[U - 1][0], (x[U - 1][n][2 + e] - ref[n][e]) + of_value[U - 1][1]));
            return w;
        };
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[n][e] = fmaxf(x[0][n][e], x[0][n][2 + e]);
                if (U > 1) top[n][e] = fmaxf(top[n][e], fmaxf(x[U - 1][n][e], x[U - 1][n][2 + e]));
                move |= top[n][e] - ref[n][e] > 8.f;
                if (kScaled) move |= top_product(n, e) > above[n][e] + 8.f;
            }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = top[n][e];
#pragma unroll
                    for (int k = 4; k < 32; k *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
                    m = fmaxf(ref[n][e], m);
                    const float up = m - ref[n][e];
                    float f = up == 0.f ? 1.f : exp2f(-up);
                    sum[n][e] *= f;
                    ref[n][e] = m;
                    if constexpr (kScaled) {
                        float w = top_product(n, e);
#pragma unroll
                        for (int k = 4; k < 32; k *= 2) w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, k));
                        const float old = above[n][e] - up;
                        w = m == kNothing ? 0.f : fmaxf(old, w);
                        f = w == old ? 1.f : exp2f(old - w);
                        above[n][e] = w;
                    }
#pragma unroll
                    for (int mm = 0; mm < M64; ++mm)
#pragma unroll
                        for (int i = 0; i < 4; ++i) { o[mm][i][n][e] *= f; o[mm][i][n][2 + e] *= f; }
                }
        }
#pragma unroll
        for (int v = 0; v < U; ++v) {
            // weights, as the second product's operand: keys 2 c, 2 c + 1 (+ 8) of row 8 n + g
            uint32_t w_hi[NR][2], w_lo[NR][2];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                float y[2][2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float u = x[v][n][2 * k + e] - ref[n][e], z = ex2_approx(u);
                        sum[n][e] += z;
                        y[k][e] = kScaled ? ex2_approx(u + (of_value[v][k] - (above[n][e] - kLift))) : z;
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (kScaled) {
                        w_hi[n][k] = transpose8(bits_of(__floats2half2_rn(y[k][0], y[k][1])));
                    } else {
                        const uint32_t w = bits_of(__floats2bfloat162_rn(y[k][0], y[k][1]));
                        w_hi[n][k] = transpose8(w);
                        w_lo[n][k] = transpose8(bits_of(__floats2bfloat162_rn(y[k][0] - __uint_as_float(w << 16), y[k][1] - __uint_as_float(w & 0xFFFF0000u))));
                    }
                }
            }
            bool hidden[4];                                  // values of keys that no row sees (0 times NaN is NaN)
#pragma unroll
            for (int n = 0; n < 4; ++n) hidden[n] = !kE2m1 && !all && (seen[v][n >> 1] >> (4 * (2 * c + (n & 1))) & 0xFu) == 0;
#pragma unroll
            for (int m0 = 0; m0 < M64; ++m0) {
                const int lot = m0 < D32 / 2 ? Sh::lot(m0, D32 / 2, Run<KIND>::kValueRuns) : 1;
                if (m0 % lot) continue;
                Word w[4][2];
#pragma unroll
                for (int n = 0; n < 4; ++n) {               // (a half group: what its other lanes find goes into columns that nobody reads)
                    const uint8_t* const row = tile + v * (2 * Sh::kKeyRow + 4 * Sh::kValueRow) + 2 * Sh::kKeyRow + n * Sh::kValueRow + Sh::value_at(m0, lane);
                    if (lot == 2 && kScaled) load_runs<kScaled ? 2 : 1>(row, w[n]);
                    else load_runs<1>(row, w[n]);
                }
                if (!kE2m1 && !all) {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        if (hidden[n]) w[n][0] = w[n][1] = Word{};
                }
                uint32_t f[2] = {0, 0};
                if constexpr (kE2m1) {
                    const int gr = min(2 * m0 + (lot == 2 ? g >> 1 : g >> 2), D32 - 1);
#pragma unroll
                    for (int h = 0; h < 2; ++h) f[h] = *reinterpret_cast<const uint32_t*>(&factors[warp][v][1][gr][2 * c + 8 * h]);
                }
#pragma unroll
                for (int mm = 0; mm < lot; ++mm) {
                    // op[i][h]: columns 2 i (h = 0, 2) and 2 i + 1 of the lane's run, keys 2 c, 2 c + 1 (h < 2) and 2 c + 8, 2 c + 9
                    uint32_t op[4][4];
                    if constexpr (KIND == MVLA_PAGE_ROWS) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint4 p0 = w[2 * h][mm], p1 = w[2 * h + 1][mm];
                            const uint32_t x0[4] = {p0.x, p0.y, p0.z, p0.w}, x1[4] = {p1.x, p1.y, p1.z, p1.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                op[i][2 * h] = __byte_perm(x0[i], x1[i], 0x5410);
                                op[i][2 * h + 1] = __byte_perm(x0[i], x1[i], 0x7632);
                            }
                        }
                    } else if constexpr (KIND == MVLA_PAGE_E4M3) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {    // (the two keys' bytes of two columns)
                                const uint2 p0 = w[2 * h][mm], p1 = w[2 * h + 1][mm];
                                from_e4m3(__byte_perm(i < 2 ? p0.x : p0.y, i < 2 ? p1.x : p1.y, i & 1 ? 0x7362 : 0x5140), op[i][2 * h], op[i][2 * h + 1]);
                            }
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {        // (the two keys' halves of a byte, of even and of odd columns)
                            const uint32_t p0 = w[2 * h][mm], p1 = w[2 * h + 1][mm];
                            uint32_t lo[4], hi[4];
                            from_e2m1((p0 & 0x0F0F0F0Fu) | (p1 << 4 & 0xF0F0F0F0u), lo);
                            from_e2m1((p0 >> 4 & 0x0F0F0F0Fu) | (p1 & 0xF0F0F0F0u), hi);
#pragma unroll
                            for (int i = 0; i < 4; ++i) { op[i][2 * h] = times(lo[i], f[h]); op[i][2 * h + 1] = times(hi[i], f[h]); }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int n = 0; n < NR; ++n) {
                            mma16<kScaled>(o[m0 + mm][i][n], op[i][0], op[i][1], op[i][2], op[i][3], w_hi[n][0], w_hi[n][1]);
                            if constexpr (!kScaled) mma16<false>(o[m0 + mm][i][n], op[i][0], op[i][1], op[i][2], op[i][3], w_lo[n][0], w_lo[n][1]);
                        }
                }
            }
        }
        if constexpr (kE2m1) __syncwarp();                   // (the factors are read)
    }
    // ---- the warps' sums (where the tiles were: their copies have all been waited for), then the cluster's
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 4; w < 32; w *= 2) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], w);
            if (g == 0) {
                merge_m[warp][8 * n + 2 * c + e] = ref[n][e] == kNothing ? -CUDART_INF_F : ref[n][e];
                merge_f[warp][8 * n + 2 * c + e] = above[n][e] - kLift;
                merge_l[warp][8 * n + 2 * c + e] = sum[n][e];
            }
        }
    __syncthreads();
    if (t < 8 * NR) {
        float m = merge_m[0][t], l = 0.f;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, merge_m[w][t]);
        const float base = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            l += merge_l[w][t] * exp2f(merge_m[w][t] - base);
            merge_f[w][t] = exp2f(0.5f * ((merge_m[w][t] - base) + merge_f[w][t]));      // (by halves: of values near 2^-117 it is no normal number)
        }
        cta_ml[t] = make_float2(m, l);
    }
    const bool whole = s.parts == 1;
    // elements col, col + 1 of row r's sums against reference m, whose exponentials have the sum l
    const auto give = [&](int r, int col, float y, float z, float m, float l) {
        const int i = r / group, head = hk * group + r - i * group;
        if (whole) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const int64_t at = (s.q_row + i) * a.n_heads + head;
            *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at * D + col) = __floats2bfloat162_rn(y * inv, z * inv);
            if (a.lse && col == 0) a.lse[at] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;      // ln 2
        } else {
            const int64_t at = (s.part0 + static_cast<int64_t>(part / ranks) * s.n_q + i) * a.n_heads + head;
            *reinterpret_cast<float2*>(a.part_o + at * D + col) = make_float2(y, z);
            if (col == 0) a.part_ml[at] = make_float2(m, l);
        }
    };
    float (*const merge_o)[8 * NR][D] = reinterpret_cast<float (*)[8 * NR][D]>(ring);
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int m = 0; m < M64; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (m < D32 / 2 || g < 4) {
                    *reinterpret_cast<float2*>(&merge_o[warp][8 * n + 2 * c][Sh::column(m, g) + 2 * i]) = make_float2(o[m][i][n][0], o[m][i][n][2]);
                    *reinterpret_cast<float2*>(&merge_o[warp][8 * n + 2 * c + 1][Sh::column(m, g) + 2 * i]) = make_float2(o[m][i][n][1], o[m][i][n][3]);
                }
    __syncthreads();
    const int pairs = n_rows * (D / 2);
    for (int u = t; u < pairs; u += kWarps * 32) {
        const int r = u / (D / 2), col = u % (D / 2) * 2;
        float y = 0.f, z = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 x2 = *reinterpret_cast<const float2*>(&merge_o[w][r][col]);
            const float half = merge_f[w][r];
            y = fmaf(x2.x * half, half, y);
            z = fmaf(x2.y * half, half, z);
        }
        if (ranks == 1) give(r, col, y, z, cta_ml[r].x, cta_ml[r].y);
        else *reinterpret_cast<float2*>(&merge_o[0][r][col]) = make_float2(y, z);
    }
    if (ranks == 1) return;                                  // (all CTAs of a launch alike)
    cluster_arrive_release();
    cluster_wait_acquire();
    if (t < 8 * NR * ranks) peer_ml[t / (8 * NR)][t % (8 * NR)] = ld_peer2(smem_u32(&cta_ml[t % (8 * NR)]), t / (8 * NR));
    __syncthreads();
    for (int u = rank * kWarps * 32 + t; u < pairs; u += ranks * kWarps * 32) {
        const int r = u / (D / 2), col = u % (D / 2) * 2;
        float2 x2[kMaxCluster];
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k)
            if (k < ranks) x2[k] = ld_peer2(smem_u32(&merge_o[0][r][col]), k);
        float m = -CUDART_INF_F, l = 0.f, y = 0.f, z = 0.f;
        for (int k = 0; k < ranks; ++k) m = fmaxf(m, peer_ml[k][r].x);
        const float base = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k)
            if (k < ranks) {
                const float f = exp2f(peer_ml[k][r].x - base);
                l = fmaf(peer_ml[k][r].y, f, l);
                y = fmaf(x2[k].x, f, y);
                z = fmaf(x2[k].y, f, z);
            }
        give(r, col, y, z, m, l);
    }
    cluster_arrive_release();                                // (nobody's sums are gone while another reads them)
    cluster_wait_acquire();
}

template <int KIND, int D32, int NR>
cudaError_t attend(const AttArgs& a, const PagePool& pool, cudaStream_t stream)
{
    static KernelSetup setup;
    constexpr int tiles = kWarps * kStages * Tile<KIND, D32>::kBytes, sums = kWarps * 8 * NR * D32 * 128, smem = tiles > sums ? tiles : sums;
    static_assert(smem == tiles || page_token_ctas(KIND, D32, NR) * (smem + 12 * 1024) <= 227 * 1024, "shape");
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(page_token_kernel<KIND, D32, NR>), smem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(a.cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, page_token_kernel<KIND, D32, NR>, a, pool);
}
template <int KIND, int D32>
cudaError_t by_rows(const AttArgs& a, const PagePool& pool, int rows, cudaStream_t stream)
{
    if constexpr (KIND != MVLA_PAGE_ROWS || D32 <= 6)        // (page_by_tokens)
        if (rows > 8) return attend<KIND, D32, 2>(a, pool, stream);
    return attend<KIND, D32, 1>(a, pool, stream);
}
template <int KIND>
cudaError_t by_dim(const AttArgs& a, const PagePool& pool, int rows, cudaStream_t stream)
{
    switch (a.head_dim / 32) {
    case 2: return by_rows<KIND, 2>(a, pool, rows, stream);
    case 3: return by_rows<KIND, 3>(a, pool, rows, stream);
    case 4: return by_rows<KIND, 4>(a, pool, rows, stream);
    case 5: return by_rows<KIND, 5>(a, pool, rows, stream);
    case 6: return by_rows<KIND, 6>(a, pool, rows, stream);
    case 7: return by_rows<KIND, 7>(a, pool, rows, stream);
    default: return by_rows<KIND, 8>(a, pool, rows, stream);
    }
}

}  // namespace

cudaError_t launch_page_token(int kind, const AttArgs& a, const PagePool& pool, int rows, cudaStream_t stream)
{
    return kind == MVLA_PAGE_ROWS ? by_dim<MVLA_PAGE_ROWS>(a, pool, rows, stream)
         : kind == MVLA_PAGE_E4M3 ? by_dim<MVLA_PAGE_E4M3>(a, pool, rows, stream)
                                  : by_dim<MVLA_PAGE_E2M1>(a, pool, rows, stream);
}

}  // namespace mvla
