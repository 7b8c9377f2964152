// Attention of fp32 query rows over pages by FMAs: blocks of 8 rows (query r / group, head r % group of the group) that share a key head.
//
// One pass over the keys in granules of 16, which lie on one page: a warp to every granule, with copies (keys of the next while the values of this are worked
// on), running maximum and sum of its own, so that warps wait for one another only for the queries and at the end, where their sums become the block's.  Scores: a lane has 2
// rows and 2 keys; outputs: 4 rows and 4 columns in 64, weights stored twice each for FMAs on pairs.
//
// B200: 208 rows of 8 heads of 64 behind 40, window 64, 6.3 us (a CTA's warps in step over tiles of 64 keys, as in attend_fma.cu: 16.6); one token over 300 rows 8.3 (23); over
// 60000 rows of 8 heads of 128, 32 query heads, 92 us, 5.3 TB/s (204).  1000 queries, prefill, 32 + 8 heads of 128: 338 us, bound by issue (blocks of 32 rows in step 393);
// 4096 over 16384 rows of 16 heads of 64, 9.5 ms (9.1).
#include "attend.cuh"
#include "f32x2.cuh"
#include "page.h"

namespace mvla {
namespace {

constexpr int kRows = 8, kGranule = 16, kPitch = 2 * kGranule + 4;      // (of a row of weights, each twice, and its factor)

__device__ __forceinline__ void copy16(float* dst, const float* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D32>
struct PageFmaShape {
    static constexpr int kD = D32 * 32, kNC = (D32 + 1) / 2;            // columns of a lane, in fours, 64 apart
    static constexpr int kWarps = page_fma_warps(D32), kCtas = page_fma_ctas(D32);
    static constexpr int kQPitch = kD + 4, kKeysOf = kGranule * kQPitch, kWarpFloats = kKeysOf + kGranule * kD + kRows * kPitch;
    static constexpr int kSmem = 4 * (kRows * kQPitch + kWarps * kWarpFloats);
    static_assert(kCtas * (kSmem + 2048) <= 227 * 1024 && kRows * kD <= kKeysOf, "shape");
};

template <int D32>
__global__ void __launch_bounds__(32 * PageFmaShape<D32>::kWarps, PageFmaShape<D32>::kCtas) page_fma_kernel(const __grid_constant__ AttArgs a)
{
    using Sh = PageFmaShape<D32>;
    constexpr int D = Sh::kD, NC = Sh::kNC, W = Sh::kWarps, QP = Sh::kQPitch;
    extern __shared__ __align__(16) float sm[];
    __shared__ float2 row_ml[W][kRows];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    float* const qs = sm;
    float* const ks = sm + kRows * QP + warp * Sh::kWarpFloats;
    float* const vs = ks + Sh::kKeysOf;
    float* const ps = vs + kGranule * D;

    pdl_wait();
    pdl_trigger();
    const int blk = a.n_blocks - 1 - static_cast<int>(blockIdx.x);       // (the last rows, which see the most, first)
    const AttSeq& s = a.s[seq_of_block(a, blk)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads;
    const int r_first = (blk - s.blk0) * kRows, n_rows = min(kRows, s.n_q * group - r_first), len = seq_len(a, s);
    const int lo = query_pos(a, s, len, r_first / group), hi = query_pos(a, s, len, (r_first + n_rows - 1) / group);
    const TileRange range = counted_tiles(len, lo, hi, kGranule, a.window, a.n_sink);
    const int per_split = (range.count + a.splits - 1) / a.splits;
    const int g1 = min(range.count, (static_cast<int>(blockIdx.z) + 1) * per_split);
    int g = static_cast<int>(blockIdx.z) * per_split + warp;
    // row of the first key of granule `i` among the rows [pages, kv_heads, page rows]; -1: zeros (without a table: the 64 rows' place among those that the sequence's queries see)
    const TileRange all = a.table ? TileRange{0, 0, 0} : counted_tiles(len, query_pos(a, s, len, 0), query_pos(a, s, len, s.n_q - 1), 64, a.window, a.n_sink);
    const auto look = [&](int i) -> int64_t {
        if (i >= g1) return -1;
        const int j = range.tile(i) * kGranule, tile = j / 64;
        const int page = a.table ? a.table[s.index * a.table_stride + (j >> a.page_shift)] : s.km_row + (tile < all.sinks ? tile : tile - all.first + all.sinks);
        return page >= 0 && page < a.n_pages ? ((static_cast<int64_t>(page) * a.kv_heads + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1)) : -1;
    };
    // whether every row of the block sees every key of a granule
    const auto inner = [&](int j0) { return j0 + kGranule - 1 <= lo && (hi - j0 < a.window || j0 + kGranule <= a.n_sink); };
    // rows that no query of the block sees may hold anything: zeros instead
    const auto copy = [&](float* dst, int pitch, const void* from, int i, int64_t at) {
        const int j0 = range.tile(i) * kGranule, r0 = lane / 8, c0 = lane % 8 * 4;
        const float* const src = static_cast<const float*>(from) + (at < 0 ? 0 : (at + r0) * D + c0);
        float* const to = dst + r0 * pitch + c0;
        if (at >= 0 && inner(j0)) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int x = 0; x < D32; ++x) copy16(to + 4 * k * pitch + 32 * x, src + 4 * k * D + 32 * x, true);
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool there = at >= 0 && j0 + r0 + 4 * k < len && some_sees(lo, hi, j0 + r0 + 4 * k, a.window, a.n_sink);
            const float* const row = there ? src + 4 * k * D : static_cast<const float*>(a.q);
#pragma unroll
            for (int x = 0; x < D32; ++x) copy16(to + 4 * k * pitch + 32 * x, row + 32 * x, there);
        }
    };
    const int64_t at0 = look(g);
    int64_t ahead = look(g + W);
    {
        const float* const q = static_cast<const float*>(a.q) + (s.q_row * a.n_heads + hk * group) * D;
        for (int r = t / 8; r < kRows; r += 4 * W) {
            const int i = (r_first + r) / group;
            const float* const row = r < n_rows ? q + (static_cast<int64_t>(i) * a.n_heads + (r_first + r - i * group)) * D : q;
#pragma unroll
            for (int c = t % 8 * 4; c < D; c += 32) copy16(qs + r * QP + c, row + c, r < n_rows);
        }
    }
    if (g < g1) copy(ks, QP, a.k, g, at0);
    copies_issued();
    if (g < g1) copy(vs, D, a.v, g, at0);
    copies_issued();

    const int kg = lane & 7, rg = lane >> 3, cg = lane & 15, rh = lane >> 4;
    int p[2];
    float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = rg + 4 * i < n_rows ? query_pos(a, s, len, (r_first + rg + 4 * i) / group) : -1;
    uint64_t o[4][NC][2] = {};
    wait_copies<1>();
    __syncthreads();                                         // the queries are there, and this warp's keys
    while (g < g1) {
        const int j0 = range.tile(g) * kGranule, next = g + W;
        uint64_t acc[2][2] = {};
#pragma unroll 8
        for (int c = 0; c < D; c += 4) {
            ulonglong2 x[2], y[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = *reinterpret_cast<const ulonglong2*>(qs + (rg + 4 * i) * QP + c);
                y[i] = *reinterpret_cast<const ulonglong2*>(ks + (kg + 8 * i) * QP + c);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = fma_f32x2(x[i].y, y[j].y, fma_f32x2(x[i].x, y[j].x, acc[i][j]));
        }
        __syncwarp();                                        // nobody reads the keys any more
        if (next < g1) copy(ks, QP, a.k, next, ahead);
        copies_issued();
        const int64_t at = ahead;
        ahead = look(next + W);
        const bool unmasked = inner(j0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float even, odd;
                split_f32(acc[i][j], even, odd);
                x[j] = unmasked || sees(p[i], j0 + kg + 8 * j, a.window, a.n_sink) ? (even + odd) * a.scale_log2 : -CUDART_INF_F;
            }
            float top = fmaxf(x[0], x[1]);
#pragma unroll
            for (int w = 4; w >= 1; w /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            top = fmaxf(m[i], top);
            const float ref = top == -CUDART_INF_F ? 0.f : top, f = exp2f(m[i] - ref);        // 0 where there was nothing yet
            float* const row = ps + (rg + 4 * i) * kPitch;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[j] = exp2f(x[j] - ref);
                sum += x[j];
                *reinterpret_cast<float2*>(row + 2 * (kg + 8 * j)) = make_float2(x[j], x[j]);
            }
            if (kg == 0) row[2 * kGranule] = f;
            m[i] = top;
            l[i] = l[i] * f + sum;                           // (this lane's keys)
        }
        wait_copies<1>();
        __syncwarp();                                        // the values are there, and the weights
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = ps[(4 * rh + i) * kPitch + 2 * kGranule];
            const uint64_t f2 = two_f32(f, f);
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) o[i][n][e] = mul_f32x2(o[i][n][e], f2);
        }
#pragma unroll
        for (int j = 0; j < kGranule; j += 2) {
            ulonglong2 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const ulonglong2*>(ps + (4 * rh + i) * kPitch + 2 * j);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const int col = D % 64 == 0 || n + 1 < NC || cg < 8 ? cg * 4 + 64 * n : 0;
                const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(vs + j * D + col), z = *reinterpret_cast<const ulonglong2*>(vs + (j + 1) * D + col);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[i][n][0] = fma_f32x2(w[i].y, z.x, fma_f32x2(w[i].x, y.x, o[i][n][0]));
                    o[i][n][1] = fma_f32x2(w[i].y, z.y, fma_f32x2(w[i].x, y.y, o[i][n][1]));
                }
            }
        }
        __syncwarp();                                        // nobody reads the values and the weights any more
        if (next < g1) copy(vs, D, a.v, next, at);
        copies_issued();
        wait_copies<1>();
        __syncwarp();                                        // the next keys are there
        g = next;
    }
    wait_copies<0>();
    // ---- the warps' sums become the block's
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int w = 4; w >= 1; w /= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        if (kg == 0) row_ml[warp][rg + 4 * i] = make_float2(m[i], l[i]);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int col = cg * 4 + 64 * n;
            if (col < D) *reinterpret_cast<ulonglong2*>(ks + (4 * rh + i) * D + col) = make_ulonglong2(o[i][n][0], o[i][n][1]);
        }
    __syncthreads();
    const bool whole = a.splits == 1;
    for (int x = t; x < n_rows * (D / 4); x += 32 * W) {
        const int r = x / (D / 4), c = x % (D / 4) * 4, rr = r_first + r, query = rr / group, h = hk * group + rr % group;
        float top = -CUDART_INF_F, sum = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, row_ml[w][r].x);
        const float ref = top == -CUDART_INF_F ? 0.f : top;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = exp2f(row_ml[w][r].x - ref);
            const float4 z = *reinterpret_cast<const float4*>(sm + kRows * QP + w * Sh::kWarpFloats + r * D + c);
            sum = fmaf(row_ml[w][r].y, f, sum);
            y.x = fmaf(z.x, f, y.x);
            y.y = fmaf(z.y, f, y.y);
            y.z = fmaf(z.z, f, y.z);
            y.w = fmaf(z.w, f, y.w);
        }
        const float f = whole ? (sum > 0.f ? 1.f / sum : 0.f) : 1.f;
        const int64_t part = (s.part0 + static_cast<int64_t>(blockIdx.z) * s.n_q + query) * a.n_heads + h;
        float* const out = whole ? static_cast<float*>(a.out) + ((s.q_row + query) * a.n_heads + h) * D : a.part_o + part * D;
        *reinterpret_cast<float4*>(out + c) = make_float4(y.x * f, y.y * f, y.z * f, y.w * f);
        if (c != 0) continue;
        if (!whole) a.part_ml[part] = make_float2(top, sum);
        else if (a.lse) a.lse[(s.q_row + query) * a.n_heads + h] = sum > 0.f ? (top + log2f(sum)) * 0.69314718055994531f : -CUDART_INF_F;      // ln 2
    }
}

template <int D32>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    using Sh = PageFmaShape<D32>;
    const cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(page_fma_kernel<D32>), Sh::kSmem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits));
    cfg.blockDim = dim3(32 * Sh::kWarps);
    cfg.dynamicSmemBytes = Sh::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, page_fma_kernel<D32>, a);
}

}  // namespace

cudaError_t launch_page_fma(const AttArgs& a, cudaStream_t stream)
{
    switch (a.head_dim / 32) {
    case 2: return attend<2>(a, stream);
    case 3: return attend<3>(a, stream);
    case 4: return attend<4>(a, stream);
    case 5: return attend<5>(a, stream);
    case 6: return attend<6>(a, stream);
    case 7: return attend<7>(a, stream);
    default: return attend<8>(a, stream);
    }
}

}  // namespace mvla
