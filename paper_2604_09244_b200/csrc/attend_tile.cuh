// What the attention kernels by tiles of 128 query rows and 64 keys share: descriptors and instructions of the tensor cores, which tiles somebody sees, and
// waits that end.
#pragma once

#include "attend.cuh"
#include "f32x2.cuh"
#include "tmem_ld.cuh"
#include "tmem_plan.h"
#include "tmem_st.cuh"

#include <cuda_fp16.h>

namespace mvla {

constexpr int kRows = 128;                   // query rows of a tile
constexpr int kKeys = 64;                    // keys of a tile
constexpr int kMaxStages = 6;
constexpr float kMoveAt = 8.f;               // a row's maximum may lie this far (powers of two) above its reference

// D[tmem] (+)= A[tmem] * B[smem], bf16, fp32 accumulate; issued by one thread.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// Shared-memory matrix descriptor of a tile whose rows (128 bytes, 128-byte swizzle) are the contraction: 64 elements of the other
// dimension lie in a row, the next 64 `box` bytes further on, the next 8 rows 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_rows_sw128(uint32_t addr, uint32_t box)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(box >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
// Instruction descriptor of fp16 or bf16 operands (format codes 0 and 1 of both), M = 128, N = n.
template <bool F16>
__device__ __forceinline__ uint32_t idesc_16(int n) { return F16 ? idesc_bf16_m128(n) & ~((1u << 7) | (1u << 10)) : idesc_bf16_m128(n); }
constexpr uint32_t kRowsAreContraction = 1u << 16;      // instruction descriptor: B as above

// Two neighbouring values of a 16-bit type: bf16, and beside what came from 8 or 4 bits (exactly) fp16, whose weights are finer.
__device__ __forceinline__ uint32_t two_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x)
{
    *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
}

// The lowest n of 32 bits (all of them from 32 on, none below 1).
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }

// What a tile of keys (or queries) is to a CTA: some row sees some key, not every row sees every key.
constexpr int kNeed = 1, kMask = 2, kEntryShift = 2;         // an entry of a list: the tile's place in the range above the flags
// Positions of `n` keys from row j0 on, by one warp: smallest and largest of those somebody may see, and whether there are others.
struct Span {
    int lo, hi;
    bool hidden;
};
__device__ __forceinline__ Span key_span(const AttArgs& a, const AttSeq& s, int len, int j0, int n, int lane)
{
    int lo = 0x7FFFFFFF, hi = -1;
    bool hidden = false;
    for (int e = lane; e < n; e += 32) {
        const int c = key_pos(a, s, len, j0 + e);
        if (c < 0) hidden = true;
        else { lo = min(lo, c); hi = max(hi, c); }
    }
    return {__reduce_min_sync(0xffffffffu, lo), __reduce_max_sync(0xffffffffu, hi), __any_sync(0xffffffffu, hidden) != 0};
}
__device__ __forceinline__ Span counted_span(int len, int j0, int n)
{
    return {j0 < len ? j0 : 0x7FFFFFFF, j0 < len ? min(j0 + n, len) - 1 : -1, j0 + n > len};
}
// Whether rows with positions in [lo, hi] see something of a span, and whether all of them see all of it.
__device__ __forceinline__ int span_flags(const AttArgs& a, int lo, int hi, const Span& k)
{
    if (k.hi < 0 || k.lo > hi || !(k.hi >= lo || lo - k.hi < a.window || k.lo < a.n_sink)) return 0;
    const bool all = k.hi <= lo && !k.hidden && (hi - k.lo < a.window || k.hi < a.n_sink);
    return all ? kNeed : kNeed | kMask;
}
// The entries with a flag among `n` flag words, in order, in place; by one warp.  Returns how many.
__device__ __forceinline__ int compact_entries(uint16_t* list, int n, int lane)
{
    int count = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int f = i0 + lane < n ? list[i0 + lane] : 0;
        const unsigned on = __ballot_sync(0xffffffffu, (f & kNeed) != 0);
        __syncwarp();
        if (f & kNeed) list[count + __popc(on & ((1u << lane) - 1u))] = static_cast<uint16_t>((i0 + lane) << kEntryShift | f);
        __syncwarp();
        count += __popc(on);
    }
    return count;
}

// Bounded waits of a CTA: when one runs out, the others end without waiting for long, and warps that meet one another go on meeting
// (attend_walk.h).  Before the CTA ends, the loads and the MMAs that are under way do: also with a limit.
struct Guard {
    int* dead;
    int* status;
    // by a whole warp: the same answer in all its lanes
    __device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)); }
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity)
    {
        if (mbar_try_wait<false>(bar, parity)) return true;
        return !*reinterpret_cast<volatile int*>(dead) && spin(bar, parity);
    }
    // of what is under way, whoever gave up
    __device__ __forceinline__ void settle(uint32_t bar, uint32_t parity)
    {
        if (!mbar_try_wait<false>(bar, parity)) spin(bar, parity);
    }
    __device__ __forceinline__ bool spin(uint32_t bar, uint32_t parity)
    {
        // (the clock of the multiprocessor, about a second of it; the global timer takes a microsecond to read)
        const long long t0 = clock64();
        for (uint32_t it = 1; it < kSpinLimit; ++it) {
            if (mbar_try_wait<false>(bar, parity)) return true;
            if ((it & 63u) == 0 && clock64() - t0 > 2000000000ll) break;
        }
        *reinterpret_cast<volatile int*>(dead) = 1;
        *reinterpret_cast<volatile int*>(status) = MVLA_ERR_TIMEOUT;
        return false;
    }
};

// ---- parts of a block of rows joined inside a cluster

__device__ __forceinline__ int cluster_ctas()
{
    int n;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
    return n;
}
// From the shared memory of CTA `rank` of this cluster, at the offset of `addr`.
__device__ __forceinline__ float2 ld_peer2(uint32_t addr, int rank)
{
    uint32_t remote;
    float2 x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(remote) : "memory");
    return x;
}
__device__ __forceinline__ float4 ld_peer4(uint32_t addr, int rank)
{
    uint32_t remote;
    float4 x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(remote) : "memory");
    return x;
}
// Where four elements, `piece` of a row's fours, lie among a CTA's sums, in fours: eight rows side by side, or eight pieces, share no bank.
__device__ __forceinline__ int sums_at(int row, int piece, int head_dim) { return row * (head_dim / 4) + (piece ^ (row & 7)); }
constexpr int kJoinFloats = kRows / 2 * (kMaxCluster + 2);               // of `factors`, for a tile of rows

// Fours of elements of `rows` rows from `first` on, added up over the R CTAs of a cluster; `give` takes them.  A thread has 16 loads on the way (a load of a peer's memory takes
// 700 cycles and more: with one four at a time the join of two CTAs' 128 rows of 128 was 2.3 us).
template <int R, class Give>
__device__ __forceinline__ void join_pieces(uint32_t sums, const float* factors, int rows, int first, int head_dim, Give give)
{
    constexpr int U = 16 / R;
    const int pieces = head_dim / 4, all = rows * pieces, step = static_cast<int>(blockDim.x);
#pragma unroll 1
    for (int u0 = threadIdx.x; u0 < all; u0 += U * step) {
        float4 x[U][R];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = min(u0 + j * step, all - 1), mine = u / pieces;
            const uint32_t at = sums + 16u * sums_at(first + mine, u - mine * pieces, head_dim);
#pragma unroll
            for (int k = 0; k < R; ++k) x[j][k] = ld_peer4(at, k);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = u0 + j * step, mine = u / pieces;
            if (u >= all) break;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float f = factors[mine * kMaxCluster + k];
                o.x = fmaf(x[j][k].x, f, o.x);
                o.y = fmaf(x[j][k].y, f, o.y);
                o.z = fmaf(x[j][k].z, f, o.z);
                o.w = fmaf(x[j][k].w, f, o.w);
            }
            give(mine, u - mine * pieces, o);
        }
    }
}
// By all threads of every CTA of a cluster (a barrier of the cluster before and behind): the sums of T tiles of rows at `sums` (sums_at), and their references and sums of
// exponentials, [T 128] at `ml`, of all its CTAs.  A CTA joins a share of the rows, in the CTAs' order: factors first, then a thread four elements of a row at a time.
template <int T>
__device__ __forceinline__ void join_cluster(const AttArgs& a, const AttSeq& s, uint32_t sums, uint32_t ml, float* factors, int ranks, int q0, int per, int head0, int part)
{
    const int t = threadIdx.x, rows = T * kRows / ranks, first = static_cast<int>(cluster_ctarank()) * rows, D = a.head_dim;
    const bool whole = s.parts == 1;
    // the query of a row of the tiles (negative: nobody's), and where its results lie, in heads
    const auto query = [&](int row) {
        const int r = row % kRows, i = q0 + row / kRows * per + r / a.pack;
        return r < per * a.pack && i < s.n_q ? i : -1;
    };
    const auto place = [&](int row, int i) {
        return (whole ? s.q_row + i : s.part0 + static_cast<int64_t>(part) * s.n_q + i) * a.n_heads + head0 + row % kRows % a.pack;
    };
    if (t < rows) {
        const int row = first + t, i = query(row);
        float2 z[kMaxCluster];
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k)
            if (k < ranks) z[k] = ld_peer2(ml + 8u * row, k);
        float m = -CUDART_INF_F, l = 0.f, f[kMaxCluster];
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k)
            if (k < ranks) m = fmaxf(m, z[k].x);
        const float ref = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k) {
            f[k] = k < ranks ? exp2f(z[k].x - ref) : 0.f;
            if (k < ranks) l = fmaf(z[k].y, f[k], l);
        }
        const float by = whole ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k)
            if (k < ranks) factors[t * kMaxCluster + k] = f[k];
        factors[rows * kMaxCluster + t] = by;
        if (i >= 0) {
            if (!whole) a.part_ml[place(row, i)] = make_float2(m, l);
            else if (a.lse) a.lse[place(row, i)] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;      // ln 2
        }
    }
    __syncthreads();
    const auto give = [&](int mine, int piece, float4 o) {
        const int row = first + mine, i = query(row);
        if (i < 0) return;
        const float by = factors[rows * kMaxCluster + mine];
        const int64_t to = place(row, i) * D + 4 * piece;
        if (whole) *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to) = make_uint2(two_bf16(o.x * by, o.y * by), two_bf16(o.z * by, o.w * by));
        else *reinterpret_cast<float4*>(a.part_o + to) = o;
    };
    if (ranks == 2) join_pieces<2>(sums, factors, rows, first, D, give);
    else if (ranks == 4) join_pieces<4>(sums, factors, rows, first, D, give);
    else join_pieces<8>(sums, factors, rows, first, D, give);
}

}  // namespace mvla
