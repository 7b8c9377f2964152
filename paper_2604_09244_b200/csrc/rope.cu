// Norms of queries and keys for each head and the position rotation, in one pass over the projections' rows.
//
//   y = x / sqrt(mean x^2 + eps) * weight;   (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = pos * inv_freq
//
// Bound by bytes: every element is read once and written once.  A CTA has one row of the batch (all its heads), so that a
// row's rot_dim / 2 angles are taken once, in 64 bits, and serve its q and k heads; a group of lanes has one head, with
// both elements of every pair in the lane that rotates them, so that nothing but the sum of squares crosses lanes.  All that does not
// depend on something else is on its way from the start (position, weights, the first heads), the next heads while one is worked on.
#include "device_utils.cuh"
#include "serve.h"

#include <cuda_fp8.h>

namespace mvla {
namespace {

constexpr int kRopeThreads = 256;

struct alignas(16) Vec16 { uint32_t w[4]; };

// Eight elements as they lie in memory, as fp32, and back (rounded once; e4m3 saturates).
template <class T> struct Raw8;
template <> struct Raw8<float> {
    float4 x, y;
    __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const float4*>(p); y = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ void get(float (&v)[8]) const { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w; }
};
template <> struct Raw8<__nv_bfloat16> {
    Vec16 r;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *reinterpret_cast<const Vec16*>(p); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
        }
    }
};
__device__ __forceinline__ void store8(float* p, const float (&x)[8])
{
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8])
{
    Vec16 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        v.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<Vec16*>(p) = v;
}
__device__ __forceinline__ void store8(__nv_fp8_e4m3* p, const float (&x)[8])
{
    uint2 v = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i], x[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        (i < 2 ? v.x : v.y) |= two << (16 * (i & 1));
    }
    *reinterpret_cast<uint2*>(p) = v;
}

template <class TIn, class TOut>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ RopeJob job)
{
    __shared__ float2 turn[128];                 // (cos, sin) of the row's angles
    const int d = job.head_dim, half = job.rot_dim / 2;
    const int units = d / 16;                    // pieces of two times eight elements in a head
    int lanes = 4;                               // lanes of a head: the next power of two
    while (lanes < units) lanes *= 2;
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x;
    const int sub = threadIdx.x % lanes, per_block = kRopeThreads / lanes;
    const bool on = sub < units;
    // this lane's two pieces of every head: a pair of halves, or 16 neighbours
    const bool rotated = 16 * sub < job.rot_dim;
    const bool halves = rotated && !job.interleaved;
    const int at0 = halves ? 8 * sub : 16 * sub, at1 = halves ? half + 8 * sub : 16 * sub + 8;
    const int n_q = job.q ? job.n_heads : 0, n_k = job.k ? job.kv_heads : 0, n_v = job.v ? job.kv_heads : 0, total = n_q + n_k + n_v;
    const TIn* const src_q = static_cast<const TIn*>(job.q) + row * job.q_stride;
    const TIn* const src_k = static_cast<const TIn*>(job.k) + row * job.k_stride;
    const TIn* const src_v = static_cast<const TIn*>(job.v) + row * job.v_stride;
    const auto what_of = [&](int h) { return h < n_q ? 0 : h < n_q + n_k ? 1 : 2; };
    const auto head_of = [&](int h, int what) { return h - (what == 0 ? 0 : what == 1 ? n_q : n_q + n_k); };
    Raw8<TIn> next0 = {}, next1 = {};
    const auto fetch = [&](int h) {
        if (!on || h >= total) return;
        const int what = what_of(h);
        const TIn* const p = (what == 0 ? src_q : what == 1 ? src_k : src_v) + static_cast<int64_t>(head_of(h, what)) * d;
        next0.load(p + at0);
        next1.load(p + at1);
    };
    int h = static_cast<int>(threadIdx.x) / lanes;
    fetch(h);
    Raw8<TIn> wq0 = {}, wq1 = {}, wk0 = {}, wk1 = {};
    const TIn* const w_q = static_cast<const TIn*>(job.q_weight);
    const TIn* const w_k = static_cast<const TIn*>(job.k_weight);
    if (on && w_q) { wq0.load(w_q + at0); wq1.load(w_q + at1); }
    if (on && w_k) { wk0.load(w_k + at0); wk1.load(w_k + at1); }
    const int64_t kv_row = job.out_rows ? job.out_rows[row] : row;
    const bool kv_there = kv_row >= 0 && kv_row < job.kv_rows;
    if (half) {
        // The angle in turns, its whole turns taken off in 64 bits: what is left is exact enough for 32.
        const double pos = job.pos[row];
        for (int i = threadIdx.x; i < half; i += kRopeThreads) {
            const double turns = pos * (job.inv_freq[i] * 0.15915494309189535);      // 1 / (2 pi)
            float s, c;
            sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
            turn[i] = make_float2(c, s);
        }
        __syncthreads();
    }
    for (int base = 0; base < total; base += per_block, h += per_block) {
        const int what = what_of(h);
        const bool live = on && h < total;
        float a[8], b[8];
        next0.get(a);
        next1.get(b);
        fetch(h + per_block);
        if (job.norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(a[i], a[i], fmaf(b[i], b[i], sum));
            if (!live) sum = 0.f;
            for (int o = lanes / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (live && what < 2) {
                const float r = 1.f / sqrtf(sum / static_cast<float>(d) + job.eps);
                float wa[8], wb[8];
                const Raw8<TIn> w0 = what == 0 ? wq0 : wk0, w1 = what == 0 ? wq1 : wk1;
                w0.get(wa);
                w1.get(wb);
                const bool weighted = (what == 0 ? w_q : w_k) != nullptr;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = a[i] * r * (weighted ? wa[i] : 1.f);
                    b[i] = b[i] * r * (weighted ? wb[i] : 1.f);
                }
            }
        }
        if (live && what < 2 && rotated) {
            if (halves) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 t = turn[8 * sub + i];
                    const float x = a[i], y = b[i];
                    a[i] = x * t.x - y * t.y;
                    b[i] = y * t.x + x * t.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 t = turn[8 * sub + i], u = turn[8 * sub + 4 + i];
                    const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
                    a[2 * i] = x * t.x - y * t.y;
                    a[2 * i + 1] = y * t.x + x * t.y;
                    b[2 * i] = z * u.x - w * u.y;
                    b[2 * i + 1] = w * u.x + z * u.y;
                }
            }
        }
        if (live && (what == 0 || kv_there)) {
            TOut* const out = static_cast<TOut*>(what == 0 ? job.q_out : what == 1 ? job.k_out : job.v_out);
            TOut* const dst = out + ((what == 0 ? row * job.n_heads : kv_row * job.kv_heads) + head_of(h, what)) * d;
            store8(dst + at0, a);
            store8(dst + at1, b);
        }
    }
}

template <class TIn, class TOut>
cudaError_t launch(const RopeJob& job, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(job.n_rows));
    cfg.blockDim = dim3(kRopeThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<TIn, TOut>, job);
}

}  // namespace

cudaError_t launch_qk_norm_rope(int dtype, const RopeJob& job, cudaStream_t stream)
{
    if (job.n_rows == 0) return cudaSuccess;
    if (dtype == MVLA_DTYPE_FP32) return launch<float, float>(job, stream);
    if (dtype == MVLA_DTYPE_BF16) return launch<__nv_bfloat16, __nv_bfloat16>(job, stream);
    return launch<__nv_bfloat16, __nv_fp8_e4m3>(job, stream);
}

}  // namespace mvla
