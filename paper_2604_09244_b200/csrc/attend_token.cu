// Windowed attention of single tokens over a cache: at most 16 query rows of a sequence share a key head (bf16, e4m3).
//
// Bound by the bytes of the keys and values.  A warp takes tiles of 16 keys as the registers that the tensor cores read (m16n8k16): keys
// are the 16 rows of the first product and columns of the values those of the second, query rows the 8 columns of both, so that a single
// token wastes as little as can be.  Which element of the head meets which is free as long as queries and keys agree, so a lane's 16 bytes
// of a key row are two steps' operands as they come, and the same holds for the columns of the values.  So every lane copies its own bytes,
// three tiles ahead, into places of its own in shared memory (asynchronously), and no lane reads another's: no barrier between the
// warps, and none between the lanes.  The scores become the second product's operand by transposing 8 x 8 blocks between the lanes.
// The sums are taken against a reference per row that is moved when some score lies 2^8 above it: one vote a tile, and no shuffle
// but then and at the end.  bf16 weights meet the values in two parts, what the type holds and what it leaves (the tensor cores have
// nothing else to do), so that rounding them costs nothing; fp16 is fine enough.
// A sequence's visible keys are cut into parts of about the same length over the whole batch; a CTA is four warps that take the part's
// tiles in turn.  With accumulated weights the scores are kept (a fraction 2 / head_dim of the keys' and values' bytes and one more for
// every query row) and become weights once all parts are joined.
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
    using Raw = uint4;                           // eight elements as they lie in memory
    static constexpr bool kTwoParts = true;
    static __device__ __forceinline__ Raw load(const __nv_bfloat16* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
    static __device__ __forceinline__ void words(const Raw& r, uint32_t (&w)[4]) { w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w; }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    static __device__ __forceinline__ float2 value(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct Kind<__nv_fp8_e4m3> {         // widened to fp16, which holds every e4m3 number
    using Raw = uint2;
    static constexpr bool kTwoParts = false;
    static __device__ __forceinline__ Raw load(const __nv_fp8_e4m3* p) { return __ldg(reinterpret_cast<const uint2*>(p)); }
    static __device__ __forceinline__ uint32_t two(uint32_t x)
    {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(x), __NV_E4M3);
        return static_cast<uint32_t>(h.x) | static_cast<uint32_t>(h.y) << 16;
    }
    static __device__ __forceinline__ void words(const Raw& r, uint32_t (&w)[4])
    {
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

// Pieces of a lane in a tile: its chunks of two key rows and of four value rows.
template <class T, int D32>
struct TokenShape {
    static constexpr int kM64 = (D32 + 1) / 2, kPieces = 2 * D32 + 4 * kM64, kPiece = 8 * sizeof(T);
    static constexpr int kTile = kPieces * 32 * kPiece;      // of a warp
    static constexpr int kSmem = kWarps * kStages * kTile, kCtas = token_ctas(D32, sizeof(T));
    static_assert(kSmem == token_smem(D32, sizeof(T)), "the plan's size");
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
    constexpr int D = D32 * 32, M64 = Sh::kM64;              // M64: groups of 64 columns of the values
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint4 q_frag[D32][NR][32];
    __shared__ float merge_o[kWarps][D];
    __shared__ float merge_m[kWarps][16], merge_l[kWarps][16];
    __shared__ int pos_ring[kWarps][kStages][32];
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, g = lane >> 2, c = lane & 3;
    const AttSeq& s = a.s[seq_of_block(a, blockIdx.x)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads, n_rows = s.n_q * group, len = seq_len(a, s);
    const T* const q = static_cast<const T*>(a.q);
    for (int u = t; u < D32 * NR * 32; u += kWarps * 32) {
        const int piece = u / (NR * 32), n = u / 32 % NR, l = u & 31, r = (l >> 2) + 8 * n;
        uint32_t w[4] = {0, 0, 0, 0};
        if (r < n_rows) K::words(K::load(q + ((s.q_row + r / group) * a.n_heads + hk * group + r % group) * D + 32 * piece + 8 * (l & 3)), w);
        q_frag[piece][n][l] = make_uint4(w[0], w[1], w[2], w[3]);
    }
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
    __syncthreads();
    const TileRange range = tile_range(a, len, lo, hi, 16);
    const int part = static_cast<int>(blockIdx.x) - s.blk0, per_part = (range.count + s.parts - 1) / s.parts;
    const int t0 = part * per_part, t1 = min(range.count, t0 + per_part);
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * D;
    const T* const kb = static_cast<const T*>(a.k) + s.kv_row * stride + static_cast<int64_t>(hk) * D + 8 * c;
    const T* const vb = static_cast<const T*>(a.v) + s.kv_row * stride + static_cast<int64_t>(hk) * D + 8 * g;
    // o[m][i][n]: columns 64 m + 8 g + 2 i and + 1 (values 0, 1 and 2, 3), rows 8 n + 2 c and + 1
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

    // Tile t0 + warp + kWarps u is this warp's u-th, in stage u % kStages.  Position of its key (lane & 15):
    const int mine = t1 > t0 + warp ? (t1 - t0 - warp + kWarps - 1) / kWarps : 0;
    const auto first_key = [&](int u) { return range.tile(t0 + warp + kWarps * u) * 16; };
    const auto pos_of = [&](int u) { return u < mine ? key_pos(a, s, len, first_key(u) + (lane & 15)) : -1; };
    const uint32_t lane_at = smem_u32(ring) + warp * kStages * Sh::kTile + lane * Sh::kPiece;
    // starts the copies of a tile that some row sees (always a group of copies, an empty one too)
    const auto fetch = [&](int u, int pos) {
        if (u < mine) {
            pos_ring[warp][u % kStages][lane] = pos;
            if (__any_sync(0xffffffffu, some_sees(lo, hi, pos, a.window, a.n_sink))) {
                const int j0 = first_key(u);
                uint32_t dst = lane_at + u % kStages * Sh::kTile;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const T* const row = kb + static_cast<int64_t>(min(j0 + 8 * n + g, len - 1)) * stride;
#pragma unroll
                    for (int i = 0; i < D32; ++i, dst += 32 * Sh::kPiece) copy_async<Sh::kPiece>(dst, row + 32 * i);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const T* const row = vb + static_cast<int64_t>(min(j0 + 2 * c + (n & 1) + 8 * (n >> 1), len - 1)) * stride;
#pragma unroll
                    for (int m = 0; m < M64; ++m, dst += 32 * Sh::kPiece)
                        if (m < D32 / 2 || g < 4) copy_async<Sh::kPiece>(dst, row + 64 * m);
                }
            }
        }
        copies_done();
    };
    int ahead[kStages - 1];
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) ahead[u] = pos_of(u);
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u, ahead[u]);
    int next = pos_of(kStages - 1);
    for (int u = 0; u < mine; ++u) {
        const int then = pos_of(u + kStages);
        fetch(u + kStages - 1, next);                        // (into the stage that the last tile was read from)
        next = then;
        wait_copies<kStages - 1>();
        const int pos = pos_ring[warp][u % kStages][lane], j0 = first_key(u);
        if (!__any_sync(0xffffffffu, some_sees(lo, hi, pos, a.window, a.n_sink))) {
            if (a.logits) {                                  // (rows that nobody sees: their weight is nothing)
                for (int rr = lane >> 1; rr < n_rows; rr += 16)
                    for (int j = j0 + 8 * (lane & 1); j < min(j0 + 8 * (lane & 1) + 8, len); ++j)
                        a.logits[s.logit0 + (static_cast<int64_t>(rr / group) * a.n_heads + hk * group + rr % group) * s.n_kv + j] = -CUDART_INF_F;
            }
            continue;
        }
        const bool all = __all_sync(0xffffffffu, pos >= 0 && pos <= lo && (hi - pos < a.window || pos < a.n_sink));
        const uint8_t* const tile = ring + (warp * kStages + u % kStages) * Sh::kTile + lane * Sh::kPiece;
        const auto piece = [&](int i) { return *reinterpret_cast<const typename K::Raw*>(tile + i * 32 * Sh::kPiece); };
        // x[n][2 k + e]: key g + 8 k, row 8 n + 2 c + e
        float x[NR][4] = {};
#pragma unroll
        for (int i = 0; i < D32; ++i) {
            uint32_t w0[4], w1[4];
            K::words(piece(i), w0);
            K::words(piece(D32 + i), w1);
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const uint4 y = q_frag[i][n][lane];
                K::mma(x[n], w0[0], w1[0], w0[1], w1[1], y.x, y.y);
                K::mma(x[n], w0[2], w1[2], w0[3], w1[3], y.z, y.w);
            }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] *= a.scale_log2;
        if (!all) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = __shfl_sync(0xffffffffu, pos, g + 8 * k);
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (!sees(p[n][e], at, a.window, a.n_sink)) x[n][2 * k + e] = -CUDART_INF_F;
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
                    for (int k = 0; k < 2; ++k)
                        if (j0 + g + 8 * k < len) dst[j0 + g + 8 * k] = x[n][2 * k + e];
                }
        }
        // references
        bool move = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) move |= fmaxf(x[n][e], x[n][2 + e]) > ref[n][e] + 8.f;
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(x[n][e], x[n][2 + e]);
#pragma unroll
                    for (int w = 4; w < 32; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                    const float m = fmaxf(ref[n][e], top), f = m == ref[n][e] ? 1.f : exp2f(ref[n][e] - m);
                    ref[n][e] = m;
                    sum[n][e] *= f;
#pragma unroll
                    for (int mm = 0; mm < M64; ++mm)
#pragma unroll
                        for (int i = 0; i < 4; ++i) { o[mm][i][n][e] *= f; o[mm][i][n][2 + e] *= f; }
                }
        }
        // weights, as the second product's operand: keys 2 c, 2 c + 1 (+ 8) of row 8 n + g
        uint32_t w_hi[NR][2], w_lo[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float b0 = ref[n][0] == -CUDART_INF_F ? 0.f : ref[n][0], b1 = ref[n][1] == -CUDART_INF_F ? 0.f : ref[n][1];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float y = ex2_approx(x[n][2 * k] - b0), z = ex2_approx(x[n][2 * k + 1] - b1);
                sum[n][0] += y;
                sum[n][1] += z;
                const uint32_t w = K::pack(y, z);
                w_hi[n][k] = transpose8(w);
                if (K::kTwoParts) {
                    const float2 v = K::value(w);
                    w_lo[n][k] = transpose8(K::pack(y - v.x, z - v.y));
                }
            }
        }
        bool hidden[4] = {};                                 // values that nobody may look at (0 times NaN is NaN)
        if (!all) {
#pragma unroll
            for (int n = 0; n < 4; ++n) hidden[n] = __shfl_sync(0xffffffffu, pos, 2 * c + (n & 1) + 8 * (n >> 1)) < 0;
        }
#pragma unroll
        for (int m = 0; m < M64; ++m) {
            uint32_t w[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                typename K::Raw v = {};
                if (!hidden[n] && (m < D32 / 2 || g < 4)) v = piece(2 * D32 + n * M64 + m);
                K::words(v, w[n]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {                    // columns 8 g + 2 i and + 1 of the group, keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
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
    // ---- the warps' sums, row by row
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 4; w < 32; w *= 2) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], w);
            if (g == 0) { merge_m[warp][8 * n + 2 * c + e] = ref[n][e]; merge_l[warp][8 * n + 2 * c + e] = sum[n][e]; }
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
                        *reinterpret_cast<float2*>(&merge_o[warp][64 * m + 8 * g + 2 * i]) = make_float2(o[m][i][r / 8][r & 1], o[m][i][r / 8][2 + (r & 1)]);
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
