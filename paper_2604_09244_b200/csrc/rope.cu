// Norms of queries and keys for each head and the position rotation, in one pass over the projections' rows.
//
//   y = x / sqrt(mean x^2 + eps) * weight;   (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = pos * inv_freq
//
// Bound by bytes: every element is read once and written once.  A CTA takes row after row of the batch (all heads of a row), so that
// what does not change with the row (weights, who has which elements) is settled once, and a row's rot_dim / 2 angles are taken
// once, in 64 bits, and serve its q and k heads; a group of lanes has one head, with both elements of every pair in the lane that rotates
// them, so that nothing but the sum of squares crosses lanes.  A row's first heads of q, k and v are on their way together.
//
// B200, bf16, 12800 rows of 32 + 32 + 32 heads of 128: 115 us (5.5 TB/s read and written; the bytes alone take 97 us).
// Arithmetic in pairs of fp32 and angles one row ahead brought it from 133 us; what is left waits for the row's loads.  Held to
// 80 registers for a third CTA on each SM it spills (144 us).  4099 rows of 32 + 8 + 8 heads of 128 to e4m3 30 us (the bytes 12): 26 of them are there
// without a rotation, since of a row's key and value heads only a quarter of the threads has one, and a CTA has one row at a time; the barrier
// between a row's angles and its heads is the rest, the same for 16 rotated elements as for 128.
#include "device_utils.cuh"
#include "f32x2.cuh"
#include "serve.h"

#include <cuda_fp8.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kRopeThreads = 256;

struct alignas(16) Vec16 { uint32_t w[4]; };

// Eight elements as they lie in memory, as four fp32 pairs, and back (rounded once; e4m3 saturates).
template <class T> struct Raw8;
template <> struct Raw8<float> {
    ulonglong2 x, y;
    __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const ulonglong2*>(p); y = *reinterpret_cast<const ulonglong2*>(p + 4); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<ulonglong2*>(p) = x; *reinterpret_cast<ulonglong2*>(p + 4) = y; }
    __device__ __forceinline__ void get(uint64_t (&v)[4]) const { v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y; }
};
template <> struct Raw8<__nv_bfloat16> {
    Vec16 r;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *reinterpret_cast<const Vec16*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<Vec16*>(p) = r; }
    __device__ __forceinline__ void get(uint64_t (&v)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = two_f32(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xFFFF0000u));
    }
};
__device__ __forceinline__ void store8(float* p, const uint64_t (&x)[4])
{
    *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(x[0], x[1]);
    *reinterpret_cast<ulonglong2*>(p + 4) = make_ulonglong2(x[2], x[3]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint64_t (&x)[4])
{
    Vec16 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split_f32(x[i], lo, hi);
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        v.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<Vec16*>(p) = v;
}
__device__ __forceinline__ void store8(__nv_fp8_e4m3* p, const uint64_t (&x)[4])
{
    uint2 v = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split_f32(x[i], lo, hi);
        const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
        (i < 2 ? v.x : v.y) |= two << (16 * (i & 1));
    }
    *reinterpret_cast<uint2*>(p) = v;
}

// A head's two pieces of one lane: normed and rotated (`turned`), or as they are.
template <class TIn, class TOut>
struct Lane {
    int sub, lanes, at0, at1;                    // place in the head's group of lanes; where the pieces begin
    bool on, rotated, halves;
    float per_d, eps;
    bool norm;
    const float *cosines, *sines;

    __device__ __forceinline__ void load(Raw8<TIn> (&raw)[2], const TIn* head) const
    {
        raw[0].load(head + at0);
        raw[1].load(head + at1);
    }
    // by all lanes of a group together; `live`: the head exists, dst: null where it is not to be written
    __device__ __forceinline__ void turn(const Raw8<TIn> (&raw)[2], const Raw8<TIn> (&weight)[2], bool weighted, bool live, TOut* dst) const
    {
        uint64_t a[4], b[4];
        raw[0].get(a);
        raw[1].get(b);
        if (norm) {
            uint64_t sums = mul_f32x2(a[0], a[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) sums = fma_f32x2(a[i], a[i], sums);
#pragma unroll
            for (int i = 0; i < 4; ++i) sums = fma_f32x2(b[i], b[i], sums);
            float even, odd;
            split_f32(sums, even, odd);
            float sum = live ? even + odd : 0.f;
            for (int o = lanes / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float r = rsqrtf(fmaf(sum, per_d, eps));
            const uint64_t rr = two_f32(r, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[i] = mul_f32x2(a[i], rr); b[i] = mul_f32x2(b[i], rr); }
            if (weighted) {
                uint64_t wa[4], wb[4];
                weight[0].get(wa);
                weight[1].get(wb);
#pragma unroll
                for (int i = 0; i < 4; ++i) { a[i] = mul_f32x2(a[i], wa[i]); b[i] = mul_f32x2(b[i], wb[i]); }
            }
        }
        if (!dst) return;
        if (rotated) {
            constexpr uint64_t kSigns = 0x8000000080000000ull, kLowSign = 0x80000000ull;
            if (halves) {                                    // pairs (a, b): two neighbouring ones at a time
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(cosines + 8 * sub + 2 * i), s = *reinterpret_cast<const ulonglong2*>(sines + 8 * sub + 2 * i);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint64_t x = a[i + e], y = b[i + e], cc = e ? c.y : c.x, ss = e ? s.y : s.x;
                        a[i + e] = fma_f32x2(x, cc, mul_f32x2(y, ss ^ kSigns));
                        b[i + e] = fma_f32x2(y, cc, mul_f32x2(x, ss));
                    }
                }
            } else {                                         // each pair of registers is a pair: (x, y) c + (y, x) (-s, s)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint64_t& z = i < 4 ? a[i & 3] : b[i & 3];
                    const float c = cosines[8 * sub + i], s = sines[8 * sub + i];
                    float x, y;
                    split_f32(z, x, y);
                    z = fma_f32x2(z, two_f32(c, c), mul_f32x2(two_f32(y, x), two_f32(s, s) ^ kLowSign));
                }
            }
        }
        store8(dst + at0, a);
        store8(dst + at1, b);
    }
    __device__ __forceinline__ void copy(const Raw8<TIn> (&raw)[2], TOut* dst) const
    {
        if constexpr (std::is_same_v<TIn, TOut>) {
            raw[0].store(dst + at0);
            raw[1].store(dst + at1);
        } else {
            uint64_t a[4], b[4];
            raw[0].get(a);
            raw[1].get(b);
            store8(dst + at0, a);
            store8(dst + at1, b);
        }
    }
};

template <class TIn, class TOut>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ RopeJob job)
{
    __shared__ __align__(16) float turn_c[2][128], turn_s[2][128];       // cosines and sines of a row's angles; rows take them in turn
    const int d = job.head_dim, half = job.rot_dim / 2, units = d / 16;  // units: pieces of two times eight elements in a head
    Lane<TIn, TOut> me;
    me.lanes = units <= 4 ? 4 : units <= 8 ? 8 : 16;                     // of a head
    me.sub = threadIdx.x % me.lanes;
    me.on = me.sub < units;
    // this lane's two pieces of every head: a pair of halves, or 16 neighbours
    me.rotated = 16 * me.sub < job.rot_dim;
    me.halves = me.rotated && !job.interleaved;
    me.at0 = me.halves ? 8 * me.sub : 16 * me.sub;
    me.at1 = me.halves ? half + 8 * me.sub : 16 * me.sub + 8;
    me.per_d = 1.f / static_cast<float>(d);
    me.eps = job.eps;
    me.norm = job.norm;
    const int h0 = static_cast<int>(threadIdx.x) / me.lanes, per_block = kRopeThreads / me.lanes;
    pdl_wait();
    pdl_trigger();
    Raw8<TIn> wq[2] = {}, wk[2] = {};
    if (me.on && job.q_weight) me.load(wq, static_cast<const TIn*>(job.q_weight));
    if (me.on && job.k_weight) me.load(wk, static_cast<const TIn*>(job.k_weight));
    const double freq = threadIdx.x < static_cast<unsigned>(half) ? job.inv_freq[threadIdx.x] * 0.15915494309189535 : 0.0;      // 1 / (2 pi)
    const int n_q = job.q ? job.n_heads : 0, n_k = job.k ? job.kv_heads : 0, n_v = job.v ? job.kv_heads : 0;
    // The angles in turns, their whole turns taken off in 64 bits: what is left is exact enough for 32.
    const auto angles = [&](int64_t row, int at) {
        if (threadIdx.x >= static_cast<unsigned>(half) || row >= job.n_rows) return;
        const double turns = job.pos[row] * freq;
        sincospif(2.f * static_cast<float>(turns - rint(turns)), &turn_s[at][threadIdx.x], &turn_c[at][threadIdx.x]);
    };
    angles(blockIdx.x, 0);
    int buf = 0;
    for (int64_t row = blockIdx.x; row < job.n_rows; row += gridDim.x, buf ^= 1) {
        const TIn* const q = static_cast<const TIn*>(job.q) + row * job.q_stride;
        const TIn* const k = static_cast<const TIn*>(job.k) + row * job.k_stride;
        const TIn* const v = static_cast<const TIn*>(job.v) + row * job.v_stride;
        Raw8<TIn> xq[2] = {}, xk[2] = {}, xv[2] = {};
        if (me.on && h0 < n_q) me.load(xq, q + h0 * d);
        if (me.on && h0 < n_k) me.load(xk, k + h0 * d);
        if (me.on && h0 < n_v) me.load(xv, v + h0 * d);
        const int64_t kv_row = job.out_rows ? job.out_rows[row] : row;
        const bool kv_there = kv_row >= 0 && kv_row < job.kv_rows;
        if (half) {
            __syncthreads();                                 // (this row's angles are there, and nobody reads the last row's any more)
            angles(row + gridDim.x, buf ^ 1);
        }
        me.cosines = turn_c[buf];
        me.sines = turn_s[buf];
        TOut* const out_q = static_cast<TOut*>(job.q_out) + row * job.n_heads * d;
        TOut* const out_k = static_cast<TOut*>(job.k_out) + kv_row * job.kv_heads * d;
        TOut* const out_v = static_cast<TOut*>(job.v_out) + kv_row * job.kv_heads * d;
        for (int base = 0, h = h0; base < n_q; base += per_block, h += per_block) {
            const bool live = me.on && h < n_q;
            if (base && live) me.load(xq, q + h * d);
            me.turn(xq, wq, job.q_weight != nullptr, live, live ? out_q + h * d : nullptr);
        }
        for (int base = 0, h = h0; base < n_k; base += per_block, h += per_block) {
            const bool live = me.on && h < n_k;
            if (base && live) me.load(xk, k + h * d);
            me.turn(xk, wk, job.k_weight != nullptr, live, live && kv_there ? out_k + h * d : nullptr);
        }
        for (int base = 0, h = h0; base < n_v; base += per_block, h += per_block) {
            if (!me.on || h >= n_v || !kv_there) continue;
            if (base) me.load(xv, v + h * d);
            me.copy(xv, out_v + h * d);
        }
    }
}

template <class TIn, class TOut>
cudaError_t launch(const RopeJob& job, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>(job.n_rows, sm_count_of_current_device() * 4)));
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
