// What follows the attention kernels: parts of a split key range joined, and weights added into the accumulated weight of every
// cached row.
#include "attend.cuh"

namespace mvla {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMassKeys = 128;               // keys of a CTA (AttSeq::tile0 counts such tiles)
constexpr int kRowGroups = kThreads / kMassKeys;
constexpr int kFinishRows = 4 * kWarps;      // rows (queries and heads) whose scores are added up at a time: eight lanes to a row's parts

__device__ __forceinline__ void store_two(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
__device__ __forceinline__ void store_two(__nv_bfloat16* p, float x, float y) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(x, y); }

// Of one (query, head), by `lanes` neighbouring lanes of a warp: the largest reference of its parts, and the sum against it.
template <int LANES>
__device__ __forceinline__ float2 parts_sum(const AttArgs& a, int64_t first, int64_t step, int parts, int lane)
{
    float m = -CUDART_INF_F;
#pragma unroll 4
    for (int p = lane; p < parts; p += LANES) m = fmaxf(m, a.part_ml[first + p * step].x);
#pragma unroll
    for (int o = LANES / 2; o >= 1; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -CUDART_INF_F ? 0.f : m;
    float l = 0.f;
#pragma unroll 4
    for (int p = lane; p < parts; p += LANES) {
        const float2 ml = a.part_ml[first + p * step];
        l += ml.y * exp2f(ml.x - ref);
    }
#pragma unroll
    for (int o = LANES / 2; o >= 1; o /= 2) l += __shfl_xor_sync(0xffffffffu, l, o);
    return make_float2(m, l);
}
__device__ __forceinline__ void write_sums(const AttArgs& a, int64_t row, int64_t unit, int h, float2 ml)
{
    const float z = ml.y > 0.f ? ml.x + log2f(ml.y) : -CUDART_INF_F;
    if (a.lse) a.lse[row * a.n_heads + h] = z * 0.69314718055994531f;      // ln 2
    if (a.lse2) a.lse2[unit] = z;
}

// x += elements c .. c + 3 of a part's sums, taken to the common reference.
__device__ __forceinline__ void add_part(const AttArgs& a, int64_t part, int c, float ref, float4& x)
{
    const float f = exp2f(a.part_ml[part].x - ref);
    const float4 o = *reinterpret_cast<const float4*>(a.part_o + part * a.head_dim + c);
    x.x = fmaf(o.x, f, x.x);
    x.y = fmaf(o.y, f, x.y);
    x.z = fmaf(o.z, f, x.z);
    x.w = fmaf(o.w, f, x.w);
}

// Few parts: a warp joins those of one (query, head), four neighbouring elements of the head to a lane at a time.  Bound by the parts' bytes.
template <class TOut>
__device__ __forceinline__ void join_by_warp(const AttArgs& a, int64_t unit)
{
    const int lane = threadIdx.x & 31;
    if (unit >= static_cast<int64_t>(a.total_q) * a.n_heads) return;
    const int qp = static_cast<int>(unit / a.n_heads), h = static_cast<int>(unit % a.n_heads);
    const AttSeq& s = a.s[seq_of_query(a, qp)];
    if (a.skip_whole && s.parts == 1) return;                // (written already)
    const int64_t row = s.q_row + (qp - s.qp0), step = static_cast<int64_t>(s.n_q) * a.n_heads, first = (s.part0 + (qp - s.qp0)) * a.n_heads + h;
    const float2 ml = parts_sum<32>(a, first, step, s.parts, lane);
    const float ref = ml.x == -CUDART_INF_F ? 0.f : ml.x, inv = ml.y > 0.f ? 1.f / ml.y : 0.f;
    for (int c = 4 * lane; c < a.head_dim; c += 128) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < s.parts; ++p) add_part(a, first + p * step, c, ref, x);
        TOut* const out = static_cast<TOut*>(a.out) + (row * a.n_heads + h) * a.head_dim + c;
        store_two(out, x.x * inv, x.y * inv);
        store_two(out + 2, x.z * inv, x.w * inv);
    }
    if (lane == 0) write_sums(a, row, unit, h, ml);
}

// Many parts: a CTA joins them, warp w the parts w, w + 8, ...; the warps' sums meet in shared memory, in order.
template <class TOut>
__device__ __forceinline__ void join_by_cta(const AttArgs& a, int64_t unit)
{
    __shared__ float sums[kWarps][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int qp = static_cast<int>(unit / a.n_heads), h = static_cast<int>(unit % a.n_heads);
    const AttSeq& s = a.s[seq_of_query(a, qp)];
    if (a.skip_whole && s.parts == 1) return;
    const int64_t row = s.q_row + (qp - s.qp0), step = static_cast<int64_t>(s.n_q) * a.n_heads, first = (s.part0 + (qp - s.qp0)) * a.n_heads + h;
    const float2 ml = parts_sum<32>(a, first, step, s.parts, lane);
    const float ref = ml.x == -CUDART_INF_F ? 0.f : ml.x, inv = ml.y > 0.f ? 1.f / ml.y : 0.f;
    for (int c = 4 * lane; c < a.head_dim; c += 128) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = warp; p < s.parts; p += kWarps) add_part(a, first + p * step, c, ref, x);
        *reinterpret_cast<float4*>(&sums[warp][c]) = x;
    }
    __syncthreads();
    for (int c = 2 * static_cast<int>(threadIdx.x); c < a.head_dim; c += 2 * kThreads) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { x += sums[w][c]; y += sums[w][c + 1]; }
        store_two(static_cast<TOut*>(a.out) + (row * a.n_heads + h) * a.head_dim + c, x * inv, y * inv);
    }
    if (threadIdx.x == 0) write_sums(a, row, unit, h, ml);
}

template <class TOut>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(const __grid_constant__ AttArgs a)
{
    pdl_wait();
    pdl_trigger();
    join_by_warp<TOut>(a, static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5));
}

template <class TOut>
__global__ void __launch_bounds__(kThreads) attend_join_cta_kernel(const __grid_constant__ AttArgs a)
{
    pdl_wait();
    pdl_trigger();
    join_by_cta<TOut>(a, blockIdx.x);
}

// What follows the kernel of single tokens: its first `joins` CTAs join parts, the others make the scores that were kept of 128 keys into
// weights and add them up, queries and heads in their order (two threads to a key, every second row each).
__global__ void __launch_bounds__(kThreads) attend_finish_kernel(const __grid_constant__ AttArgs a, int joins)
{
    __shared__ float row_z[2][kFinishRows], half[kMassKeys];
    pdl_wait();
    pdl_trigger();
    if (static_cast<int>(blockIdx.x) < joins) {
        if (a.splits > kFewParts) join_by_cta<__nv_bfloat16>(a, blockIdx.x);
        else join_by_warp<__nv_bfloat16>(a, static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5));
        return;
    }
    const int tile = static_cast<int>(blockIdx.x) - joins, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const AttSeq& s = a.s[seq_at(a, tile, [](const AttSeq& x) { return x.tile0; })];
    if (s.n_q == 0) return;
    const int len = seq_len(a, s), j = (tile - s.tile0) * kMassKeys + t % kMassKeys, group = t / kMassKeys;
    bool seen = j < len;
    if (seen && !a.kv_pos) {                                 // (counted positions: keys outside the window were not looked at and have no score)
        int lo = 0x7FFFFFFF, hi = -1;
        for (int i = 0; i < s.n_q; ++i) {
            const int p = query_pos(a, s, len, i);
            lo = min(lo, p);
            hi = max(hi, p);
        }
        seen = some_sees(lo, hi, j, a.window, a.n_sink);
    }
    if (!__syncthreads_or(seen)) return;
    const int rows = s.n_q * a.n_heads;
    const float* const x = a.logits + s.logit0 + j;
    float sum = 0.f;
    for (int r0 = 0, buf = 0; r0 < rows; r0 += kFinishRows, buf ^= 1) {
        float y[kFinishRows / kRowGroups];                   // the scores, on their way with the parts' sums
#pragma unroll
        for (int i = 0; i < kFinishRows / kRowGroups; ++i) {
            const int r = r0 + group + i * kRowGroups;
            y[i] = seen && r < rows ? x[static_cast<int64_t>(r) * s.n_kv] : -CUDART_INF_F;
        }
        {                                                    // the logarithm of a row's sum by eight lanes
            const int r = warp * 4 + (lane >> 3), mine = min(r0 + r, rows - 1);
            const float2 ml = parts_sum<8>(a, s.part0 * a.n_heads + mine, rows, s.parts, lane & 7);
            if ((lane & 7) == 0) row_z[buf][r] = ml.y > 0.f ? ml.x + log2f(ml.y) : 0.f;
        }
        __syncthreads();                                     // (and nobody is with the buffer that is written next)
#pragma unroll
        for (int i = 0; i < kFinishRows / kRowGroups; ++i) sum += exp2f(y[i] - row_z[buf][group + i * kRowGroups]);      // (2^-inf is 0)
    }
    if (group == 1) half[t % kMassKeys] = sum;
    __syncthreads();
    if (group == 0 && seen) {
        sum += half[t];
        if (sum != 0.f) a.mass[s.kv_row + j] += sum / static_cast<float>(a.n_heads);
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
#pragma unroll 8
    for (int h = 0; h < a.mass_parts; ++h) sum += a.part_mass[static_cast<int64_t>(h) * a.total_kv + at];
    if (sum != 0.f) a.mass[s.kv_row + j] += sum / static_cast<float>(a.n_heads);
}

template <class K, class... Args>
cudaError_t launch(K kernel, int64_t blocks, cudaStream_t stream, Args... args)
{
    if (blocks == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t launch_attend_join(int dtype, bool by_ctas, const AttArgs& a, cudaStream_t stream)
{
    const int64_t units = static_cast<int64_t>(a.total_q) * a.n_heads, blocks = (units + kWarps - 1) / kWarps;
    if (by_ctas)
        return dtype == MVLA_DTYPE_FP32 ? launch(attend_join_cta_kernel<float>, units, stream, a) : launch(attend_join_cta_kernel<__nv_bfloat16>, units, stream, a);
    return dtype == MVLA_DTYPE_FP32 ? launch(attend_join_kernel<float>, blocks, stream, a) : launch(attend_join_kernel<__nv_bfloat16>, blocks, stream, a);
}

cudaError_t launch_attend_finish(const AttArgs& a, cudaStream_t stream)
{
    const int64_t units = a.splits > 1 ? static_cast<int64_t>(a.total_q) * a.n_heads : 0;
    const int64_t joins = a.splits > kFewParts ? units : (units + kWarps - 1) / kWarps;
    const AttSeq& last = a.s[a.n_seq - 1];
    const int64_t tiles = a.mass ? last.tile0 + (last.n_kv + kMassKeys - 1) / kMassKeys : 0;
    return launch(attend_finish_kernel, joins + tiles, stream, a, static_cast<int>(joins));
}

cudaError_t launch_mass_add(const AttArgs& a, cudaStream_t stream)
{
    return launch(mass_add_kernel, (static_cast<int64_t>(a.total_kv) + kThreads - 1) / kThreads, stream, a);
}

}  // namespace mvla
