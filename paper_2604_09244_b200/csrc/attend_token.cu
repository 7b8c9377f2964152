// Windowed attention of single tokens over a cache: at most 16 query rows of a sequence share a key head (bf16, e4m3).
//
// Bound by the bytes of the keys and values.  A warp takes tiles of 16 keys as the registers that the tensor cores read (m16n8k16, rows x
// keys x head): which element of the head meets which is free as long as queries and keys agree, so a lane's 16 bytes of a key row are two
// steps' operands as they come, and the same holds for the columns of the values.  So every lane copies its own bytes, three tiles
// ahead, into places of its own in shared memory (asynchronously), and no lane reads another's: no barrier between the warps, and none
// between the lanes.  The scores' registers are the weights' registers of the second product.
// The sums are taken against a reference per row that is moved when some score lies 2^8 above it: one vote a tile, and no shuffle
// between rows and lanes but then and at the end.  Weights meet the values in two parts, what the 16-bit type holds and what it leaves
// (the tensor cores have nothing else to do), so that rounding them costs nothing.
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

// D32: pieces of 32 elements in a head.  BOTH: more than eight query rows.
template <class T, int D32, bool BOTH>
__global__ void __launch_bounds__(kWarps * 32, TokenShape<T, D32>::kCtas) attend_token_kernel(const __grid_constant__ AttArgs a)
{
    using K = Kind<T>;
    constexpr int D = D32 * 32, M64 = (D32 + 1) / 2;         // M64: groups of 64 columns of the values
    constexpr int kHalves = BOTH ? 2 : 1;                    // rows g and g + 8 of a lane
    using Sh = TokenShape<T, D32>;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ int pos_ring[kWarps][kStages][32];
    __shared__ uint4 q_frag[D32][kHalves][32];
    __shared__ float merge_o[kWarps][D];
    __shared__ float merge_m[kWarps][16], merge_l[kWarps][16];
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, g = lane >> 2, c = lane & 3;
    const AttSeq& s = a.s[seq_of_block(a, blockIdx.x)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads, n_rows = s.n_q * group, len = seq_len(a, s);
    const T* const q = static_cast<const T*>(a.q);
    for (int u = t; u < D32 * kHalves * 32; u += kWarps * 32) {
        const int piece = u / (kHalves * 32), h = u / 32 % kHalves, l = u & 31, r = (l >> 2) + 8 * h;
        uint32_t w[4] = {0, 0, 0, 0};
        if (r < n_rows) K::words(K::load(q + ((s.q_row + r / group) * a.n_heads + hk * group + r % group) * D + 32 * piece + 8 * (l & 3)), w);
        q_frag[piece][h][l] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    int p[kHalves], lo = 0x7FFFFFFF, hi = -1;                // this lane's rows, and the span of all rows
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        const int r = g + 8 * h;
        p[h] = r < n_rows ? query_pos(a, s, len, r / group) : -1;
        if (r < n_rows) { lo = min(lo, p[h]); hi = max(hi, p[h]); }
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
    float o[M64][8][4];
#pragma unroll
    for (int m = 0; m < M64; ++m)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[m][i][0] = o[m][i][1] = o[m][i][2] = o[m][i][3] = 0.f;
    float ref[kHalves], sum[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) { ref[h] = -CUDART_INF_F; sum[h] = 0.f; }

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
        float x[2][4] = {};
#pragma unroll
        for (int i = 0; i < D32; ++i) {
            const uint4 qa = q_frag[i][0][lane];
            const uint4 qb = BOTH ? q_frag[i][kHalves - 1][lane] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                uint32_t w[4];
                K::words(piece(n * D32 + i), w);
                K::mma(x[n], qa.x, qb.x, qa.y, qb.y, w[0], w[1]);
                K::mma(x[n], qa.z, qb.z, qa.w, qb.w, w[2], w[3]);
            }
        }
        // x[n][2 h + e]: row g + 8 h, key 8 n + 2 c + e
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] *= a.scale_log2;
        if (!all) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int k = __shfl_sync(0xffffffffu, pos, 8 * n + 2 * c + e);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (h >= kHalves || !sees(p[h < kHalves ? h : 0], k, a.window, a.n_sink)) x[n][2 * h + e] = -CUDART_INF_F;
                }
        }
        if (a.logits) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const int r = g + 8 * h;
                if (r >= n_rows) continue;
                float* const dst = a.logits + s.logit0 + (static_cast<int64_t>(r / group) * a.n_heads + hk * group + r % group) * s.n_kv;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int j = j0 + 8 * n + 2 * c + e;
                        if (j < len) dst[j] = x[n][2 * h + e];
                    }
            }
        }
        // references
        bool move = false;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const float top = fmaxf(fmaxf(x[0][2 * h], x[0][2 * h + 1]), fmaxf(x[1][2 * h], x[1][2 * h + 1]));
            move |= top > ref[h] + 8.f;
        }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                float top = fmaxf(fmaxf(x[0][2 * h], x[0][2 * h + 1]), fmaxf(x[1][2 * h], x[1][2 * h + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const float m = fmaxf(ref[h], top);
                const float f = m == ref[h] ? 1.f : exp2f(ref[h] - m);
                ref[h] = m;
                sum[h] *= f;
#pragma unroll
                for (int mm = 0; mm < M64; ++mm)
#pragma unroll
                    for (int i = 0; i < 8; ++i) { o[mm][i][2 * h] *= f; o[mm][i][2 * h + 1] *= f; }
            }
        }
        uint32_t w_hi[4] = {0, 0, 0, 0}, w_lo[4] = {0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const float base = ref[h] == -CUDART_INF_F ? 0.f : ref[h];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float y = ex2_approx(x[n][2 * h] - base), z = ex2_approx(x[n][2 * h + 1] - base);
                sum[h] += y + z;
                const uint32_t w = K::pack(y, z);
                const float2 v = K::value(w);
                w_hi[2 * n + h] = w;
                w_lo[2 * n + h] = K::pack(y - v.x, z - v.y);
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
            for (int i = 0; i < 8; ++i) {                    // column 8 g + i of the group, keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
                const uint32_t sel = i & 1 ? 0x7632u : 0x5410u;
                const uint32_t b0 = __byte_perm(w[0][i / 2], w[1][i / 2], sel), b1 = __byte_perm(w[2][i / 2], w[3][i / 2], sel);
                K::mma(o[m][i], w_hi[0], w_hi[1], w_hi[2], w_hi[3], b0, b1);
                K::mma(o[m][i], w_lo[0], w_lo[1], w_lo[2], w_lo[3], b0, b1);
            }
        }
    }
    // ---- the warps' sums, row by row
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        if (c == 0) { merge_m[warp][g + 8 * h] = ref[h]; merge_l[warp][g + 8 * h] = sum[h]; }
    }
    const bool whole = s.parts == 1;
    for (int r = 0; r < n_rows; ++r) {
        __syncthreads();
        if (g == (r & 7)) {
#pragma unroll
            for (int m = 0; m < M64; ++m)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int col = 64 * m + 16 * c + 8 * e + i;
                        const float v = BOTH && r >= 8 ? o[m][i][2 + e] : o[m][i][e];
                        if (col < D) merge_o[warp][col] = v;
                    }
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
            if (whole) {
                const float z = l > 0.f ? m + log2f(l) : -CUDART_INF_F;
                if (a.lse) a.lse[(s.q_row + i) * a.n_heads + head] = z * 0.69314718055994531f;      // ln 2
            }
            if (a.part_ml) a.part_ml[at] = make_float2(m, l);
        }
    }
}

template <class T, int D32, bool BOTH>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(attend_token_kernel<T, D32, BOTH>), TokenShape<T, D32>::kSmem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = TokenShape<T, D32>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_token_kernel<T, D32, BOTH>, a);
}
template <class T, int D32>
cudaError_t by_rows(const AttArgs& a, int rows, cudaStream_t stream)
{
    return rows <= 8 ? attend<T, D32, false>(a, stream) : attend<T, D32, true>(a, stream);
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
