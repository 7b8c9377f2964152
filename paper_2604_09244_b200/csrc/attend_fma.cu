// Windowed attention by FMAs in 32 bits, and the weights that it gives to the cached rows.
//
// Flash form: one pass over the keys in tiles of 64, running maximum and sum per query row, exponentials in powers of two.  A CTA
// has a block of query rows that share a key head: row r of a block is query r / group, head r % group of the group, so that a
// single token's grouped heads share the keys they read.
#include "attend.cuh"

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p)
{
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
}
__device__ __forceinline__ float4 load4(const __nv_fp8_e4m3* p) { return make_float4(float(p[0]), float(p[1]), float(p[2]), float(p[3])); }
__device__ __forceinline__ void store4(float* p, const float4& x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float4& x)
{
    reinterpret_cast<__nv_bfloat162*>(p)[0] = __floats2bfloat162_rn(x.x, x.y);
    reinterpret_cast<__nv_bfloat162*>(p)[1] = __floats2bfloat162_rn(x.z, x.w);
}
template <class T> struct OutOf { using type = __nv_bfloat16; };
template <> struct OutOf<float> { using type = float; };

// n rows of one key head, `stride` elements apart, into shared memory with `pitch` floats a row; rows from
// `valid` on, and those of negative position where `pos` says so, become zero.
template <class T>
__device__ __forceinline__ void load_rows(float* dst, int pitch, const T* src, int64_t stride, int n, int valid, int d, const int* pos)
{
    const int per = d / 4;
    for (int u = threadIdx.x; u < n * per; u += kThreads) {
        const int r = u / per, c = u - r * per;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < valid && pos[r] >= 0) x = load4(src + r * stride + c * 4);
        *reinterpret_cast<float4*>(dst + r * pitch + c * 4) = x;
    }
}

// RT x KT dot products of this thread: rows r0 + i, keys k0 + j (64 / KT apart).
template <int RT, int KT>
__device__ __forceinline__ void dots(float (&acc)[RT][KT], const float* q, const float* k, int q_pitch, int k_pitch, int d)
{
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < KT; ++j) acc[i][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < d; c += 4) {
        float4 x[RT], y[KT];
#pragma unroll
        for (int i = 0; i < RT; ++i) x[i] = *reinterpret_cast<const float4*>(q + i * q_pitch + c);
#pragma unroll
        for (int j = 0; j < KT; ++j) y[j] = *reinterpret_cast<const float4*>(k + j * (kTile / KT) * k_pitch + c);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
                acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
                acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
                acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
            }
    }
}

size_t fma_smem(int rows, int d) { return sizeof(float) * (static_cast<size_t>(rows) * d + kTile * (d + 4) + kTile * d + rows * kTile + 4 * rows + kTile); }

template <class T, int R>
__global__ void __launch_bounds__(kThreads) attend_fma_kernel(const __grid_constant__ AttArgs a)
{
    constexpr int RT = R / 16 > 0 ? R / 16 : 1;              // rows of a thread in the dot products
    constexpr int KT = kTile * R / RT / kThreads;            // keys
    constexpr int TK = kTile / KT;                           // threads side by side over the keys
    constexpr int PER = kThreads / R;                        // threads of a row in its statistics
    constexpr int MAXU = R / 4;                              // rows of a thread in the output (at least four threads over the rows)
    extern __shared__ __align__(16) float sm[];
    const int d = a.head_dim, c4 = d / 4;
    float* const qs = sm;
    float* const ks = qs + R * d;
    float* const vs = ks + kTile * (d + 4);
    float* const ps = vs + kTile * d;
    float* const row_m = ps + R * kTile;
    float* const row_l = row_m + R;
    float* const row_f = row_l + R;
    int* const row_p = reinterpret_cast<int*>(row_f + R);
    int* const pos = row_p + R;

    pdl_wait();
    pdl_trigger();
    const int b = seq_of_block(a, blockIdx.x);
    const AttSeq& s = a.s[b];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads;
    const int r_first = (static_cast<int>(blockIdx.x) - s.blk0) * R, n_rows = min(R, s.n_q * group - r_first);
    const int len = seq_len(a, s);
    const int t = threadIdx.x;
    const T* const q = static_cast<const T*>(a.q);
    for (int u = t; u < R * c4; u += kThreads) {
        const int r = u / c4, c = u - r * c4, rr = r_first + r;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < n_rows) x = load4(q + ((s.q_row + rr / group) * a.n_heads + hk * group + rr % group) * d + c * 4);
        *reinterpret_cast<float4*>(qs + r * d + c * 4) = x;
    }
    if (t < R) {
        row_m[t] = -CUDART_INF_F;
        row_l[t] = 0.f;
        row_p[t] = t < n_rows ? query_pos(a, s, len, (r_first + t) / group) : -1;
    }
    __syncthreads();
    int lo = 0x7FFFFFFF, hi = -1;                            // (positions below zero see nothing)
    for (int r = 0; r < n_rows; ++r)
        if (row_p[r] >= 0) { lo = min(lo, row_p[r]); hi = max(hi, row_p[r]); }
    const TileRange range = tile_range(a, len, lo, hi, kTile);
    const int per_split = (range.count + a.splits - 1) / a.splits;
    const int t0 = static_cast<int>(blockIdx.z) * per_split, t1 = min(range.count, t0 + per_split);

    const int tr2 = kThreads / c4, orow = t / c4, ocol = (t % c4) * 4;
    const bool owner = t < c4 * tr2;
    float o[MAXU][4];
#pragma unroll
    for (int n = 0; n < MAXU; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * d;
    const T* const k = static_cast<const T*>(a.k) + s.kv_row * stride + static_cast<int64_t>(hk) * d;
    const T* const v = static_cast<const T*>(a.v) + s.kv_row * stride + static_cast<int64_t>(hk) * d;
    for (int it = t0; it < t1; ++it) {
        const int j0 = range.tile(it) * kTile, valid = min(kTile, len - j0);
        bool any = false;
        if (t < kTile) {
            const int c = key_pos(a, s, len, j0 + t);
            pos[t] = c;
            any = some_sees(lo, hi, c, a.window, a.n_sink);
        }
        if (!__syncthreads_or(any)) continue;
        load_rows(ks, d + 4, k + j0 * stride, stride, kTile, valid, d, pos);
        load_rows(vs, d, v + j0 * stride, stride, kTile, valid, d, pos);
        __syncthreads();
        const int rq = t / TK * RT, kq = t % TK;
        float acc[RT][KT];
        dots<RT, KT>(acc, qs + rq * d, ks + kq * (d + 4), d, d + 4, d);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < KT; ++j)
                ps[(rq + i) * kTile + kq + j * TK] = sees(row_p[rq + i], pos[kq + j * TK], a.window, a.n_sink) ? acc[i][j] * a.scale_log2 : -CUDART_INF_F;
        __syncthreads();
        {
            const int r = t / PER, c = t % PER;
            float top = -CUDART_INF_F;
            for (int j = c; j < kTile; j += PER) top = fmaxf(top, ps[r * kTile + j]);
#pragma unroll
            for (int w = PER / 2; w >= 1; w /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float old = row_m[r], m = fmaxf(old, top);
            const float ref = m == -CUDART_INF_F ? 0.f : m;
            float sum = 0.f;
            for (int j = c; j < kTile; j += PER) {
                const float p = exp2f(ps[r * kTile + j] - ref);
                ps[r * kTile + j] = p;
                sum += p;
            }
#pragma unroll
            for (int w = PER / 2; w >= 1; w /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            __syncwarp();
            if (c == 0) {
                const float f = exp2f(old - ref);            // 0 where there was nothing yet
                row_f[r] = f;
                row_m[r] = m;
                row_l[r] = row_l[r] * f + sum;
            }
        }
        __syncthreads();
        if (owner) {
#pragma unroll
            for (int n = 0; n < MAXU; ++n) {
                const int r = orow + n * tr2;
                if (r < R) {
                    const float f = row_f[r];
                    o[n][0] *= f; o[n][1] *= f; o[n][2] *= f; o[n][3] *= f;
                }
            }
            for (int j = 0; j < kTile; ++j) {
                const float4 x = *reinterpret_cast<const float4*>(vs + j * d + ocol);
#pragma unroll
                for (int n = 0; n < MAXU; ++n) {
                    const int r = orow + n * tr2;
                    if (r < R) {
                        const float p = ps[r * kTile + j];
                        o[n][0] = fmaf(p, x.x, o[n][0]);
                        o[n][1] = fmaf(p, x.y, o[n][1]);
                        o[n][2] = fmaf(p, x.z, o[n][2]);
                        o[n][3] = fmaf(p, x.w, o[n][3]);
                    }
                }
            }
        }
        __syncthreads();
    }
    const bool whole = a.splits == 1;
    if (owner) {
#pragma unroll
        for (int n = 0; n < MAXU; ++n) {
            const int r = orow + n * tr2, rr = r_first + r;
            if (r >= n_rows) continue;
            const int i = rr / group, h = hk * group + rr % group;
            const float l = row_l[r], f = whole ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
            const float4 x = make_float4(o[n][0] * f, o[n][1] * f, o[n][2] * f, o[n][3] * f);
            if (whole) store4(static_cast<typename OutOf<T>::type*>(a.out) + ((s.q_row + i) * a.n_heads + h) * d + ocol, x);
            else store4(a.part_o + ((s.part0 + static_cast<int64_t>(blockIdx.z) * s.n_q + i) * a.n_heads + h) * d + ocol, x);
        }
    }
    if (t < n_rows) {
        const int rr = r_first + t, i = rr / group, h = hk * group + rr % group;
        if (whole) {
            const float z = row_l[t] > 0.f ? row_m[t] + log2f(row_l[t]) : -CUDART_INF_F;
            if (a.lse) a.lse[(s.q_row + i) * a.n_heads + h] = z * 0.69314718055994531f;      // ln 2
            if (a.mass) a.lse2[static_cast<int64_t>(s.qp0 + i) * a.n_heads + h] = z;
        } else {
            a.part_ml[(s.part0 + static_cast<int64_t>(blockIdx.z) * s.n_q + i) * a.n_heads + h] = make_float2(row_m[t], row_l[t]);
        }
    }
}

size_t mass_smem(int d) { return sizeof(float) * (32u * d + kTile * (d + 4) + 32 * kTile + 2 * 32 + kTile); }

// One CTA: 64 cached rows of a sequence, one key head; its queries in blocks of 32 rows, in order.
template <class T>
__global__ void __launch_bounds__(kThreads) mass_fma_kernel(const __grid_constant__ AttArgs a)
{
    constexpr int R = 32, RT = 2, KT = 4, TK = kTile / KT;
    extern __shared__ __align__(16) float sm[];
    const int d = a.head_dim, c4 = d / 4;
    float* const qs = sm;
    float* const ks = qs + R * d;
    float* const ps = ks + kTile * (d + 4);
    float* const row_z = ps + R * kTile;
    int* const row_p = reinterpret_cast<int*>(row_z + R);
    int* const pos = row_p + R;
    pdl_wait();
    pdl_trigger();
    int b = 0, tile = blockIdx.x;
    while (b + 1 < a.n_seq && tile >= (a.s[b].n_kv + kTile - 1) / kTile) tile -= (a.s[b++].n_kv + kTile - 1) / kTile;
    const AttSeq& s = a.s[b];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads, t = threadIdx.x;
    const int len = seq_len(a, s), j0 = tile * kTile, valid = min(kTile, len - j0);
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * d;
    if (t < kTile) pos[t] = key_pos(a, s, len, j0 + t);
    __syncthreads();
    int c_lo = 0x7FFFFFFF, c_hi = -1;
    for (int j = 0; j < kTile; ++j)
        if (pos[j] >= 0) { c_lo = min(c_lo, pos[j]); c_hi = max(c_hi, pos[j]); }
    load_rows(ks, d + 4, static_cast<const T*>(a.k) + (s.kv_row + j0) * stride + static_cast<int64_t>(hk) * d, stride, kTile, valid, d, pos);
    float sum = 0.f;
    const int total = s.n_q * group;
    for (int r0 = 0; r0 < total && c_hi >= 0; r0 += R) {
        const int n_rows = min(R, total - r0);
        bool any = false;
        __syncthreads();
        if (t < R) {
            const int rr = r0 + t;
            const int p = t < n_rows ? query_pos(a, s, len, rr / group) : -1;
            row_p[t] = p;
            row_z[t] = t < n_rows ? a.lse2[static_cast<int64_t>(s.qp0 + rr / group) * a.n_heads + hk * group + rr % group] : 0.f;
            any = p >= c_lo && (c_lo < a.n_sink || p < c_hi || p - c_hi < a.window);
        }
        if (!__syncthreads_or(any)) continue;
        for (int u = t; u < R * c4; u += kThreads) {
            const int r = u / c4, c = u - r * c4, rr = r0 + r;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < n_rows) x = load4(static_cast<const T*>(a.q) + ((s.q_row + rr / group) * a.n_heads + hk * group + rr % group) * d + c * 4);
            *reinterpret_cast<float4*>(qs + r * d + c * 4) = x;
        }
        __syncthreads();
        const int rq = t / TK * RT, kq = t % TK;
        float acc[RT][KT];
        dots<RT, KT>(acc, qs + rq * d, ks + kq * (d + 4), d, d + 4, d);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < KT; ++j)
                ps[(rq + i) * kTile + kq + j * TK] =
                    sees(row_p[rq + i], pos[kq + j * TK], a.window, a.n_sink) ? exp2f(acc[i][j] * a.scale_log2 - row_z[rq + i]) : 0.f;
        __syncthreads();
        if (t < kTile)
            for (int r = 0; r < n_rows; ++r) sum += ps[r * kTile + t];
    }
    if (t < kTile && j0 + t < s.n_kv) a.part_mass[static_cast<int64_t>(hk) * a.total_kv + s.kvp0 + j0 + t] = sum;
}

template <class K>
cudaError_t launch(KernelSetup& setup, K kernel, dim3 grid, size_t smem, const AttArgs& a, cudaStream_t stream)
{
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(kernel), smem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class T, int R>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    return launch(setup, attend_fma_kernel<T, R>, dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits)),
                  fma_smem(R, a.head_dim), a, stream);
}

template <class T>
cudaError_t mass(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    int64_t tiles = 0;
    for (int b = 0; b < a.n_seq; ++b) tiles += (a.s[b].n_kv + kTile - 1) / kTile;
    if (tiles == 0) return cudaSuccess;
    return launch(setup, mass_fma_kernel<T>, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(a.kv_heads)), mass_smem(a.head_dim), a, stream);
}

}  // namespace

cudaError_t launch_attend_fma(int dtype, const AttArgs& a, int rows, cudaStream_t stream)
{
    if (dtype == MVLA_DTYPE_FP32) return rows == 8 ? attend<float, 8>(a, stream) : attend<float, 32>(a, stream);
    if (dtype == MVLA_DTYPE_BF16) return rows == 8 ? attend<__nv_bfloat16, 8>(a, stream) : attend<__nv_bfloat16, 32>(a, stream);
    return rows == 8 ? attend<__nv_fp8_e4m3, 8>(a, stream) : attend<__nv_fp8_e4m3, 32>(a, stream);
}

cudaError_t launch_mass_fma(int dtype, const AttArgs& a, cudaStream_t stream)
{
    if (dtype == MVLA_DTYPE_FP32) return mass<float>(a, stream);
    return dtype == MVLA_DTYPE_BF16 ? mass<__nv_bfloat16>(a, stream) : mass<__nv_fp8_e4m3>(a, stream);
}

}  // namespace mvla
