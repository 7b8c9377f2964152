// Norms of queries and keys for each head and the position rotation, in one pass over the projections' rows.
//
//   y = x / sqrt(mean x^2 + eps) * weight;   (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = pos * inv_freq
//
// Bound by bytes: every element is read once and written once.  A CTA has one row of the batch (all its heads), so that a
// row's rot_dim / 2 angles are taken once, in 64 bits, and serve its q and k heads; a group of lanes has one head, with
// both elements of every pair in the lane that rotates them, so that nothing but the sum of squares crosses lanes.
#include "device_utils.cuh"
#include "serve.h"

#include <cuda_fp8.h>

namespace mvla {
namespace {

constexpr int kRopeThreads = 256;

struct alignas(16) Vec16 { uint32_t w[4]; };

// Eight elements as fp32, and back (rounded once; e4m3 saturates).
__device__ __forceinline__ void load8(const float* p, float (&x)[8])
{
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8])
{
    const Vec16 v = *reinterpret_cast<const Vec16*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v.w[i] << 16);
        x[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u);
    }
}
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
    const int64_t kv_row = job.out_rows ? job.out_rows[row] : row;
    const bool kv_there = kv_row >= 0 && kv_row < job.kv_rows;
    const int n_q = job.q ? job.n_heads : 0, n_k = job.k && kv_there ? job.kv_heads : 0, n_v = job.v && kv_there ? job.kv_heads : 0;
    const int sub = threadIdx.x % lanes, per_block = kRopeThreads / lanes;
    const bool on = sub < units;
    // this lane's two pieces of every head: a pair of halves, or 16 neighbours
    const bool rotated = 16 * sub < job.rot_dim;
    const bool halves = rotated && !job.interleaved;
    const int at0 = halves ? 8 * sub : 16 * sub, at1 = halves ? half + 8 * sub : 16 * sub + 8;
    const int total = n_q + n_k + n_v;
    for (int base = 0; base < total; base += per_block) {
        const int h = base + static_cast<int>(threadIdx.x) / lanes;
        const int what = h < n_q ? 0 : h < n_q + n_k ? 1 : 2;
        const bool live = on && h < total;
        float a[8] = {}, b[8] = {};
        TOut* dst = nullptr;
        if (live) {
            const TIn* src;
            if (what == 0) {
                src = static_cast<const TIn*>(job.q) + row * job.q_stride + static_cast<int64_t>(h) * d;
                dst = static_cast<TOut*>(job.q_out) + (row * job.n_heads + h) * d;
            } else if (what == 1) {
                src = static_cast<const TIn*>(job.k) + row * job.k_stride + static_cast<int64_t>(h - n_q) * d;
                dst = static_cast<TOut*>(job.k_out) + (kv_row * job.kv_heads + h - n_q) * d;
            } else {
                src = static_cast<const TIn*>(job.v) + row * job.v_stride + static_cast<int64_t>(h - n_q - n_k) * d;
                dst = static_cast<TOut*>(job.v_out) + (kv_row * job.kv_heads + h - n_q - n_k) * d;
            }
            load8(src + at0, a);
            load8(src + at1, b);
        }
        if (job.norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(a[i], a[i], fmaf(b[i], b[i], sum));
            for (int o = lanes / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (live && what < 2) {
                const float r = 1.f / sqrtf(sum / static_cast<float>(d) + job.eps);
                const TIn* w = static_cast<const TIn*>(what == 0 ? job.q_weight : job.k_weight);
                float wa[8], wb[8];
                if (w) {
                    load8(w + at0, wa);
                    load8(w + at1, wb);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = a[i] * r * (w ? wa[i] : 1.f);
                    b[i] = b[i] * r * (w ? wb[i] : 1.f);
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
        if (live) {
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
