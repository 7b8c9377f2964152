// What follows the attention kernels: parts of a split key range joined, and the weights of the heads added into the
// accumulated weight of every cached row.
#include "attend.cuh"

namespace mvla {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void store_two(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
__device__ __forceinline__ void store_two(__nv_bfloat16* p, float x, float y) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(x, y); }

// A warp joins the parts of one (query, head), two neighbouring elements of the head to a lane at a time.  Bound by the parts' bytes.
template <class TOut>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(const __grid_constant__ AttArgs a)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
    if (unit >= static_cast<int64_t>(a.total_q) * a.n_heads) return;
    const int qp = static_cast<int>(unit / a.n_heads), h = static_cast<int>(unit % a.n_heads);
    const AttSeq& s = a.s[seq_of_query(a, qp)];
    const int64_t row = s.q_row + (qp - s.qp0), step = static_cast<int64_t>(s.n_q) * a.n_heads;
    const int64_t first = (s.part0 + (qp - s.qp0)) * a.n_heads + h;
    if (a.skip_whole && s.parts == 1) return;                // (written already)
    float m = -CUDART_INF_F;
    for (int p = 0; p < s.parts; ++p) m = fmaxf(m, a.part_ml[first + p * step].x);
    const float ref = m == -CUDART_INF_F ? 0.f : m;
    float l = 0.f;
    for (int p = 0; p < s.parts; ++p) {
        const float2 ml = a.part_ml[first + p * step];
        l += ml.y * exp2f(ml.x - ref);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int c = 2 * lane; c < a.head_dim; c += 64) {
        float x = 0.f, y = 0.f;
        for (int p = 0; p < s.parts; ++p) {
            const float f = exp2f(a.part_ml[first + p * step].x - ref);
            const float2 o = *reinterpret_cast<const float2*>(a.part_o + (first + p * step) * a.head_dim + c);
            x = fmaf(o.x, f, x);
            y = fmaf(o.y, f, y);
        }
        store_two(static_cast<TOut*>(a.out) + (row * a.n_heads + h) * a.head_dim + c, x * inv, y * inv);
    }
    if (lane == 0) {
        const float z = l > 0.f ? m + log2f(l) : -CUDART_INF_F;
        if (a.lse) a.lse[row * a.n_heads + h] = z * 0.69314718055994531f;      // ln 2
        if (a.mass) a.lse2[unit] = z;
    }
}

// One thread adds the parts' weights of one cached row, in their order.
__global__ void __launch_bounds__(kThreads) mass_add_kernel(const __grid_constant__ AttArgs a)
{
    pdl_wait();
    pdl_trigger();
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (at >= a.total_kv) return;
    const AttSeq& s = a.s[seq_of_key(a, static_cast<int>(at))];
    const int j = static_cast<int>(at) - s.kvp0;
    if (s.n_q == 0 || j >= seq_len(a, s)) return;
    float sum = 0.f;
    for (int h = 0; h < a.mass_parts; ++h) sum += a.part_mass[static_cast<int64_t>(h) * a.total_kv + at];
    if (sum != 0.f) a.mass[s.kv_row + j] += sum / static_cast<float>(a.n_heads);
}

template <class K>
cudaError_t launch(K kernel, int64_t blocks, const AttArgs& a, cudaStream_t stream)
{
    if (blocks == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace

cudaError_t launch_attend_join(int dtype, const AttArgs& a, cudaStream_t stream)
{
    const int64_t blocks = (static_cast<int64_t>(a.total_q) * a.n_heads + kThreads / 32 - 1) / (kThreads / 32);
    return dtype == MVLA_DTYPE_FP32 ? launch(attend_join_kernel<float>, blocks, a, stream) : launch(attend_join_kernel<__nv_bfloat16>, blocks, a, stream);
}

cudaError_t launch_mass_add(const AttArgs& a, cudaStream_t stream)
{
    return launch(mass_add_kernel, (static_cast<int64_t>(a.total_kv) + kThreads - 1) / kThreads, a, stream);
}

}  // namespace mvla
