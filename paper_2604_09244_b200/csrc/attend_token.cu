// Windowed attention of single tokens over a cache: at most 16 query rows of a sequence share a key head (e4m3; bf16 where weights are added up,
// heads have 64 elements, lengths are unlike or the call is short: by_tokens in attend_plan.h).
//
// Bound by the bytes of the keys and values.  A warp takes tiles of 16 keys as the registers that the tensor cores read (m16n8k16): keys
// are the 16 rows of the first product and columns of the values those of the second, query rows the 8 columns of both, so that a single
// token wastes as little as can be.  Which element of the head meets which is free as long as queries and keys agree, so a lane's 16 bytes
// of a key row are two steps' operands as they come, and the same holds for the columns of the values.  So every lane copies its own bytes,
// three tiles ahead, into places of its own in shared memory (asynchronously), and no lane reads another's: no barrier between the
// warps, and none between the lanes.  The scores become the second product's operand by transposing 8 x 8 blocks between the lanes.
// The sums are taken against a reference per row that is moved when some score lies 2^8 above it: one vote a tile, and no shuffle
// but then and at the end.  bf16 weights meet the values in two parts, what the type holds and what it leaves (the tensor cores have
// nothing else to do), so that rounding them costs nothing; fp16 weights (e4m3 rows) are one part, lifted (kF16Lift).
// A sequence's visible keys are cut into parts of about the same length over the whole batch; a CTA is four warps that take the part's
// tiles in turn.  With accumulated weights the scores are kept (a fraction 2 / head_dim of the keys' and values' bytes and one more for
// every query row) and become weights once all parts are joined.
//
// B200, one token each, with what follows the kernel: 16 requests over 500 to 4000 e4m3 rows of 8 heads of 128, window 2048, weights added up 43 us
// (74 MB that have to be looked at; 680 instructions of a warp to 16 keys, of which the schedulers issue 0.42 a cycle: bound by their latency, 2.7
// warps a scheduler); 60000 e4m3 rows of 32 heads 127 us, 3.9 TB/s; 16 requests over bf16 rows of 32 heads with weights 144 us, 4.1 TB/s.  Tiles of 32
// e4m3 keys halve the CTAs that fit: 47 us instead of 44 (16 requests), 133 instead of 126 (60000 rows).  (e4m3 heads of 96 with more than eight rows:
// 20 bytes spill for the fourth CTA; nowhere else.)
#include "attend.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = 3;                   // tiles of a warp in shared memory

// `BYTES` (8 or 16) from global memory to this lane's place, asynchronously; and waits for all groups of copies but the last N.
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T> struct Kind;
template <> struct Kind<__nv_bfloat16> {
    using Run = uint4;                           // eight elements as they lie in memory
    // 32 elements of 16 keys (rows g and g + 8 of a lane) with those of eight query rows
    static __device__ __forceinline__ void scores(float (&x)[4], const Run& k0, const Run& k1, const Run& y)
    {
        mma(x, k0.x, k1.x, k0.y, k1.y, y.x, y.y);
        mma(x, k0.z, k1.z, k0.w, k1.w, y.z, y.w);
    }
    static constexpr bool kTwoParts = true;
    static constexpr float kLift = 0.f;
    static constexpr bool kPairs = false;        // eight elements are what a lane copies at once
    // eight elements as the products' 16-bit pairs
    static __device__ __forceinline__ void words(const void* p, uint32_t (&w)[4])
    {
        const uint4 r = *static_cast<const uint4*>(p);
        w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    static __device__ __forceinline__ float2 value(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct Kind<__nv_fp8_e4m3> {         // scores from the 8-bit operands; values widened to fp16, which holds every e4m3 number
    using Run = uint2;
    static __device__ __forceinline__ void scores(float (&x)[4], const Run& k0, const Run& k1, const Run& y)
    {
        asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]) : "r"(k0.x), "r"(k1.x), "r"(k0.y), "r"(k1.y), "r"(y.x), "r"(y.y));
    }
    static constexpr bool kTwoParts = false;
    static constexpr float kLift = kF16Lift;
    static constexpr bool kPairs = true;         // sixteen, where a head has them
    static __device__ __forceinline__ uint32_t two(uint32_t x)
    {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(x), __NV_E4M3);
        return static_cast<uint32_t>(h.x) | static_cast<uint32_t>(h.y) << 16;
    }
    static __device__ __forceinline__ void words(const void* p, uint32_t (&w)[4])
    {
        const uint2 r = *static_cast<const uint2*>(p);
        w[0] = two(r.x & 0xFFFFu); w[1] = two(r.x >> 16); w[2] = two(r.y & 0xFFFFu); w[3] = two(r.y >> 16);
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_f16(lo, hi); }
    static __device__ __forceinline__ float2 value(uint32_t w)
    {
        const __half2 h = *reinterpret_cast<const __half2*>(&w);
        return __half22float2(h);
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

// A warp's tile of kKeys keys in shared memory: runs of 8 or 16 bytes of every lane, side by side.  A row of keys is cut into runs of eight
// elements (32 elements a step of four lanes), or of sixteen (64) where two steps make a pair; a row of values into runs of eight
// columns (64 a group of eight lanes) or sixteen (128).
template <class T, int D32>
struct TokenShape {
    static constexpr int kM64 = (D32 + 1) / 2, kSub = token_sub(D32), kKeys = 16 * kSub;
    static constexpr int kRun = 8 * sizeof(T);
    static constexpr int kKPairs = Kind<T>::kPairs ? D32 / 2 : 0, kVPairs = Kind<T>::kPairs ? D32 / 4 : 0;     // pairs of steps, of groups
    static constexpr int kKRow = D32 * 32 * kRun, kVRow = kM64 * 32 * kRun;       // of a lane's row of keys, of values, for the whole warp
    static constexpr int kTile = kSub * (2 * kKRow + 4 * kVRow);
    static constexpr int kSmem = kWarps * kStages * kTile, kCtas = token_ctas(D32, sizeof(T));
    static_assert(kSmem == token_smem(D32, sizeof(T)), "the plan's size");
    // element of the head at which lane c's run of step i begins; column at which lane g's of group m does
    static __device__ __forceinline__ int element(int i, int c) { return i < 2 * kKPairs ? 64 * (i / 2) + 16 * c + 8 * (i & 1) : 32 * i + 8 * c; }
    static __device__ __forceinline__ int column(int m, int g) { return m < 2 * kVPairs ? 128 * (m / 2) + 16 * g + 8 * (m & 1) : 64 * m + 8 * g; }
    // where they lie in a row of the tile
    static __device__ __forceinline__ int key_at(int i, int lane) { return i < 2 * kKPairs ? (i / 2) * 64 * kRun + lane * 2 * kRun + (i & 1) * kRun : i * 32 * kRun + lane * kRun; }
    static __device__ __forceinline__ int value_at(int m, int lane) { return m < 2 * kVPairs ? (m / 2) * 64 * kRun + lane * 2 * kRun + (m & 1) * kRun : m * 32 * kRun + lane * kRun; }
};

// The transpose of an 8 x 8 block of 16-bit values, a pair of neighbours in every lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// D32: pieces of 32 elements in a head.  NR: groups of eight query rows.
template <class T, int D32, int NR>
__global__ void __launch_bounds__(kWarps * 32, TokenShape<T, D32>::kCtas) attend_token_kernel(const __grid_constant__ AttArgs a)
{
    using K = Kind<T>;
    using Sh = TokenShape<T, D32>;
    constexpr int D = D32 * 32, M64 = Sh::kM64, U = Sh::kSub;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ typename K::Run q_frag[D32][NR][32];
    __shared__ float merge_o[kWarps][D];
    __shared__ float merge_m[kWarps][16], merge_l[kWarps][16];
    __shared__ int pos_ring[kWarps][kStages][32];
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, g = lane >> 2, c = lane & 3;
    const AttSeq& s = a.s[seq_of_block(a, blockIdx.x)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads, n_rows = s.n_q * group, len = seq_len(a, s);
    int p[NR][2], lo = 0x7FFFFFFF, hi = -1;                  // positions of this lane's rows 8 n + 2 c + e, and the span of all rows
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * c + e;
            p[n][e] = r < n_rows ? query_pos(a, s, len, r / group) : -1;
            if (r < n_rows) { lo = min(lo, p[n][e]); hi = max(hi, p[n][e]); }
        }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const TileRange range = tile_range(a, len, lo, hi, Sh::kKeys);
    const int part = static_cast<int>(blockIdx.x) - s.blk0, per_part = (range.count + s.parts - 1) / s.parts;
    const int t0 = part * per_part, t1 = min(range.count, t0 + per_part);
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * D;
    const T* const kb = static_cast<const T*>(a.k) + s.kv_row * stride + static_cast<int64_t>(hk) * D;
    const T* const vb = static_cast<const T*>(a.v) + s.kv_row * stride + static_cast<int64_t>(hk) * D;
    // o[m][i][n]: columns column(m, g) + 2 i and + 1 (values 0, 1 and 2, 3), rows 8 n + 2 c and + 1
    float o[M64][4][NR][4];
#pragma unroll
    for (int m = 0; m < M64; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NR; ++n) o[m][i][n][0] = o[m][i][n][1] = o[m][i][n][2] = o[m][i][n][3] = 0.f;
    float ref[NR][2], sum[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) { ref[n][0] = ref[n][1] = -CUDART_INF_F; sum[n][0] = sum[n][1] = 0.f; }

    // Tile t0 + warp + kWarps u is this warp's u-th.  Position of its key (lane % kKeys):
    const int mine = t1 > t0 + warp ? (t1 - t0 - warp + kWarps - 1) / kWarps : 0;
    const auto first_key = [&](int u) { return range.tile(t0 + warp + kWarps * u) * Sh::kKeys; };
    const auto pos_of = [&](int u) { return u < mine ? key_pos(a, s, len, first_key(u) + lane % Sh::kKeys) : -1; };
    uint8_t* const stages = ring + warp * kStages * Sh::kTile;
    const uint32_t stages_at = smem_u32(stages);
    // starts the copies of a tile that some row sees (always a group of copies, an empty one too)
    const auto fetch = [&](int u, int stage, int pos) {
        if (u < mine) {
            pos_ring[warp][stage][lane] = pos;
            if (__any_sync(0xffffffffu, some_sees(lo, hi, pos, a.window, a.n_sink))) {
                const int j0 = first_key(u);
                uint32_t dst = stages_at + stage * Sh::kTile;
#pragma unroll
                for (int n = 0; n < 2 * U; ++n, dst += Sh::kKRow) {
                    const T* const row = kb + static_cast<int64_t>(min(j0 + 8 * n + g, len - 1)) * stride;
#pragma unroll
                    for (int i = 0; i < D32; ++i) {
                        if (i < 2 * Sh::kKPairs && (i & 1)) continue;
                        if (i < 2 * Sh::kKPairs) copy_async<2 * Sh::kRun>(dst + Sh::key_at(i, lane), row + Sh::element(i, c));
                        else copy_async<Sh::kRun>(dst + Sh::key_at(i, lane), row + Sh::element(i, c));
                    }
                }
#pragma unroll
                for (int n = 0; n < 4 * U; ++n, dst += Sh::kVRow) {
                    const T* const row = vb + static_cast<int64_t>(min(j0 + 16 * (n / 4) + 2 * c + (n & 1) + 8 * (n >> 1 & 1), len - 1)) * stride;
#pragma unroll
                    for (int m = 0; m < M64; ++m) {
                        if (m < 2 * Sh::kVPairs && (m & 1)) continue;
                        if (m < 2 * Sh::kVPairs) copy_async<2 * Sh::kRun>(dst + Sh::value_at(m, lane), row + Sh::column(m, g));
                        else if (m < D32 / 2 || g < 4) copy_async<Sh::kRun>(dst + Sh::value_at(m, lane), row + Sh::column(m, g));
                    }
                }
            }
        }
        copies_done();
    };
    int ahead[kStages - 1];
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) ahead[u] = pos_of(u);
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u, u, ahead[u]);
    const T* const q = static_cast<const T*>(a.q);
    for (int u = t; u < D32 * NR * 32; u += kWarps * 32) {
        const int piece = u / (NR * 32), n = u / 32 % NR, l = u & 31, r = (l >> 2) + 8 * n;
        typename K::Run w = {};
        if (r < n_rows) w = *reinterpret_cast<const typename K::Run*>(q + ((s.q_row + r / group) * a.n_heads + hk * group + r % group) * D + Sh::element(piece, l & 3));
        q_frag[piece][n][l] = w;
    }
    __syncthreads();
    int next = pos_of(kStages - 1), stage = 0;
    for (int u = 0; u < mine; ++u, stage = stage + 1 < kStages ? stage + 1 : 0) {
        const int then = pos_of(u + kStages);
        fetch(u + kStages - 1, stage > 0 ? stage - 1 : kStages - 1, next);       // (into the stage that the last tile was read from)
        next = then;
        wait_copies<kStages - 1>();
        const int pos = pos_ring[warp][stage][lane], j0 = first_key(u);
        if (!__any_sync(0xffffffffu, some_sees(lo, hi, pos, a.window, a.n_sink))) {
            if (a.logits) {                                  // (rows that nobody sees: their weight is nothing)
                for (int r = 0; r < n_rows; ++r)
                    if (lane < Sh::kKeys && j0 + lane < len)
                        a.logits[s.logit0 + (static_cast<int64_t>(r / group) * a.n_heads + hk * group + r % group) * s.n_kv + j0 + lane] = -CUDART_INF_F;
            }
            continue;
        }
        const bool all = __all_sync(0xffffffffu, pos >= 0 && pos <= lo && (hi - pos < a.window || pos < a.n_sink));
        const uint8_t* const tile = stages + stage * Sh::kTile;
        // x[v][n][2 k + e]: key 16 v + g + 8 k, row 8 n + 2 c + e
        float x[U][NR][4] = {};
#pragma unroll
        for (int i = 0; i < D32; ++i) {
            typename K::Run y[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n) y[n] = q_frag[i][n][lane];
#pragma unroll
            for (int v = 0; v < U; ++v) {
                const auto k0 = *reinterpret_cast<const typename K::Run*>(tile + 2 * v * Sh::kKRow + Sh::key_at(i, lane));
                const auto k1 = *reinterpret_cast<const typename K::Run*>(tile + (2 * v + 1) * Sh::kKRow + Sh::key_at(i, lane));
#pragma unroll
                for (int n = 0; n < NR; ++n) K::scores(x[v][n], k0, k1, y[n]);
            }
        }
#pragma unroll
        for (int v = 0; v < U; ++v)
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[v][n][i] *= a.scale_log2;
        uint32_t seen[U][2] = {};                            // four bits for every key g + 8 k: which lanes have a row that sees it
        if (!all) {
#pragma unroll
            for (int v = 0; v < U; ++v)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = __shfl_sync(0xffffffffu, pos, 16 * v + g + 8 * k);
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
        if (a.logits) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 8 * n + 2 * c + e;
                    if (r >= n_rows) continue;
                    float* const dst = a.logits + s.logit0 + (static_cast<int64_t>(r / group) * a.n_heads + hk * group + r % group) * s.n_kv;
#pragma unroll
                    for (int k = 0; k < 2 * U; ++k)
                        if (j0 + g + 8 * k < len) dst[j0 + g + 8 * k] = x[k / 2][n][2 * (k & 1) + e];
                }
        }
        // references
        float top[NR][2];
        bool move = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[n][e] = fmaxf(x[0][n][e], x[0][n][2 + e]);
                if (U > 1) top[n][e] = fmaxf(top[n][e], fmaxf(x[U - 1][n][e], x[U - 1][n][2 + e]));
                move |= top[n][e] > ref[n][e] + 8.f;
            }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = top[n][e];
#pragma unroll
                    for (int w = 4; w < 32; w *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
                    m = fmaxf(ref[n][e], m);
                    const float f = m == ref[n][e] ? 1.f : exp2f(ref[n][e] - m);
                    ref[n][e] = m;
                    sum[n][e] *= f;
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
                const float b0 = ref[n][0] == -CUDART_INF_F ? 0.f : ref[n][0] - K::kLift, b1 = ref[n][1] == -CUDART_INF_F ? 0.f : ref[n][1] - K::kLift;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float y = ex2_approx(x[v][n][2 * k] - b0), z = ex2_approx(x[v][n][2 * k + 1] - b1);
                    sum[n][0] += y;
                    sum[n][1] += z;
                    const uint32_t w = K::pack(y, z);
                    w_hi[n][k] = transpose8(w);
                    if (K::kTwoParts) {
                        const float2 back = K::value(w);
                        w_lo[n][k] = transpose8(K::pack(y - back.x, z - back.y));
                    }
                }
            }
            bool hidden[4];                                  // values of keys that no row sees (0 times NaN is NaN)
#pragma unroll
            for (int n = 0; n < 4; ++n) hidden[n] = !all && (seen[v][n >> 1] >> (4 * (2 * c + (n & 1))) & 0xFu) == 0;
#pragma unroll
            for (int m = 0; m < M64; ++m) {
                uint32_t w[4][4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    w[n][0] = w[n][1] = w[n][2] = w[n][3] = 0;
                    if (!hidden[n] && (m < D32 / 2 || g < 4)) K::words(tile + 2 * U * Sh::kKRow + (4 * v + n) * Sh::kVRow + Sh::value_at(m, lane), w[n]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {                // columns 2 i and 2 i + 1 of the lane's run, keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
                    const uint32_t a0 = __byte_perm(w[0][i], w[1][i], 0x5410), a1 = __byte_perm(w[0][i], w[1][i], 0x7632);
                    const uint32_t a2 = __byte_perm(w[2][i], w[3][i], 0x5410), a3 = __byte_perm(w[2][i], w[3][i], 0x7632);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        K::mma(o[m][i][n], a0, a1, a2, a3, w_hi[n][0], w_hi[n][1]);
                        if (K::kTwoParts) K::mma(o[m][i][n], a0, a1, a2, a3, w_lo[n][0], w_lo[n][1]);
                    }
                }
            }
        }
    }
    // ---- the warps' sums, row by row
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 4; w < 32; w *= 2) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], w);
            if (g == 0) { merge_m[warp][8 * n + 2 * c + e] = ref[n][e] - K::kLift; merge_l[warp][8 * n + 2 * c + e] = sum[n][e]; }
        }
    const bool whole = s.parts == 1;
#pragma unroll
    for (int r = 0; r < 8 * NR; ++r) {
        if (r >= n_rows) break;
        __syncthreads();
        if (c == (r & 7) >> 1) {
#pragma unroll
            for (int m = 0; m < M64; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (m < D32 / 2 || g < 4)
                        *reinterpret_cast<float2*>(&merge_o[warp][Sh::column(m, g) + 2 * i]) = make_float2(o[m][i][r / 8][r & 1], o[m][i][r / 8][2 + (r & 1)]);
        }
        __syncthreads();
        float m = merge_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, merge_m[w][r]);
        const float base = m == -CUDART_INF_F ? 0.f : m;
        float l = 0.f, f[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            f[w] = exp2f(merge_m[w][r] - base);
            l += merge_l[w][r] * f[w];
        }
        const float inv = whole ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
        const int i = r / group, head = hk * group + r % group;
        const int64_t at = (s.part0 + static_cast<int64_t>(part) * s.n_q + i) * a.n_heads + head;
        for (int col = 2 * t; col < D; col += 2 * kWarps * 32) {
            float x = 0.f, y = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                x = fmaf(merge_o[w][col], f[w], x);
                y = fmaf(merge_o[w][col + 1], f[w], y);
            }
            if (whole) reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + ((s.q_row + i) * a.n_heads + head) * D)[col / 2] = __floats2bfloat162_rn(x * inv, y * inv);
            else *reinterpret_cast<float2*>(a.part_o + at * D + col) = make_float2(x, y);
        }
        if (t == 0) {
            if (whole && a.lse) a.lse[(s.q_row + i) * a.n_heads + head] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;      // ln 2
            if (a.part_ml) a.part_ml[at] = make_float2(m, l);
        }
    }
}

template <class T, int D32, int NR>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(attend_token_kernel<T, D32, NR>), TokenShape<T, D32>::kSmem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = TokenShape<T, D32>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_token_kernel<T, D32, NR>, a);
}
template <class T, int D32>
cudaError_t by_rows(const AttArgs& a, int rows, cudaStream_t stream)
{
    return rows <= 8 ? attend<T, D32, 1>(a, stream) : attend<T, D32, 2>(a, stream);
}
template <class T>
cudaError_t by_dim(const AttArgs& a, int rows, cudaStream_t stream)
{
    switch (a.head_dim / 32) {
    case 2: return by_rows<T, 2>(a, rows, stream);
    case 3: return by_rows<T, 3>(a, rows, stream);
    case 4: return by_rows<T, 4>(a, rows, stream);
    case 5: return by_rows<T, 5>(a, rows, stream);
    case 6: return by_rows<T, 6>(a, rows, stream);
    case 7: return by_rows<T, 7>(a, rows, stream);
    default: return by_rows<T, 8>(a, rows, stream);
    }
}

}  // namespace

cudaError_t launch_attend_token(int dtype, const AttArgs& a, int rows, cudaStream_t stream)
{
    return dtype == MVLA_DTYPE_BF16 ? by_dim<__nv_bfloat16>(a, rows, stream) : by_dim<__nv_fp8_e4m3>(a, rows, stream);
}

}  // namespace mvla
