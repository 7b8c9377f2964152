// Windowed attention of fp32 rows by FMAs, and the weights that it gives to the cached rows.
//
// One pass over the keys in tiles of 64, running maximum and sum per query row, exponentials in powers of two.  A CTA has a
// block of 32 (8) query rows that share a key head: row r of a block is query r / group, head r % group of the group.  A half warp has 4 (1)
// of them for the whole pass, in the scores and in the output, so that a row's statistics stay in its registers and its weights
// cross only the half warp; a thread works out 4 x 4 scores from 8 loads of four elements, and 4 x 4 outputs likewise, which is where the
// FMAs and the reads of shared memory are about even.  Keys and values have a buffer each: the next keys are copied while
// the values are worked on, the values while the keys are.
//
// B200: 208 rows of 8 heads of 64, window 64: 18 us (of it about 9 the launch and three tiles' latencies).  1500 rows of 32 + 8 heads of
// 128, everything before a row visible: 720 us, 26 TFLOP/s, bound by the FMAs and the reads of shared memory beside them.  One token
// over 30000 rows of 32 heads of 128: 252 us, 3.9 TB/s.  The weights of the 1500 rows: 400 us more, 1340 when every key's rows were one CTA's.
// (Blocks of 8 rows of heads above 192 elements spill 24 bytes.)
#include "attend.cuh"
#include "f32x2.cuh"

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 128;
constexpr int kTile = 64;                                    // keys
constexpr int kKeys = kTile / 16;                            // of a thread: 16 apart
constexpr int kPitch = kTile + 4;                            // floats of a row of weights

// 16 bytes into shared memory, zeros where `there` does not hold (nothing is read then).
__device__ __forceinline__ void copy16(float* dst, const float* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The tile's rows of one key head; those of negative position become zero.
__device__ __forceinline__ void copy_keys(float* dst, int pitch, const float* src, int64_t stride, int d, const int* pos)
{
    for (int r = threadIdx.x / 8; r < kTile; r += kThreads / 8) {
        const bool there = pos[r] >= 0;
        const float* const row = there ? src + r * stride : src;
        for (int c = threadIdx.x % 8 * 4; c < d; c += 32) copy16(dst + r * pitch + c, row + c, there);
    }
}
// n rows from rr on (query rr / group, head rr % group of the group) of a sequence whose queries begin at `q`; zeros up to R.
template <int R>
__device__ __forceinline__ void copy_queries(float* dst, const float* q, int rr, int n, int group, int n_heads, int d)
{
    for (int r = threadIdx.x / 8; r < R; r += kThreads / 8) {
        const int i = (rr + r) / group;
        const float* const row = r < n ? q + (static_cast<int64_t>(i) * n_heads + (rr + r - i * group)) * d : q;
        for (int c = threadIdx.x % 8 * 4; c < d; c += 32) copy16(dst + r * d + c, row + c, r < n);
    }
}

// Dot products of this thread: its RT rows from q on, keys 16 apart from k on.  Even and odd elements are summed in two halves.
template <int RT>
__device__ __forceinline__ void dots(float (&s)[RT][kKeys], const float* q, const float* k, int d)
{
    uint64_t acc[RT][kKeys] = {};
    const int pitch = d + 4;
#pragma unroll 2
    for (int c = 0; c < d; c += 4) {
        ulonglong2 x[RT], y[kKeys];
#pragma unroll
        for (int i = 0; i < RT; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(q + i * d + c);
#pragma unroll
        for (int j = 0; j < kKeys; ++j) y[j] = *reinterpret_cast<const ulonglong2*>(k + j * 16 * pitch + c);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < kKeys; ++j) acc[i][j] = fma_f32x2(x[i].y, y[j].y, fma_f32x2(x[i].x, y[j].x, acc[i][j]));
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
            float lo, hi;
            split_f32(acc[i][j], lo, hi);
            s[i][j] = lo + hi;
        }
}

size_t attend_smem(int rows, int d) { return sizeof(float) * (static_cast<size_t>(rows) * (d + kPitch) + kTile * (2 * d + 4)); }

// RT: rows of a half warp.  NC: columns of a thread, in fours, 64 apart.
template <int RT, int NC>
__global__ void __launch_bounds__(kThreads) attend_fma_kernel(const __grid_constant__ AttArgs a)
{
    constexpr int R = 8 * RT;
    extern __shared__ __align__(16) float sm[];
    __shared__ int row_p[R], pos[2][kTile];
    const int d = a.head_dim, t = threadIdx.x;
    float* const ks = sm;
    float* const vs = ks + kTile * (d + 4);
    float* const qs = vs + kTile * d;
    float* const ps = qs + R * d;

    pdl_wait();
    pdl_trigger();
    const AttSeq& s = a.s[seq_of_block(a, blockIdx.x)];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads;
    const int r_first = (static_cast<int>(blockIdx.x) - s.blk0) * R, n_rows = min(R, s.n_q * group - r_first);
    copy_queries<R>(qs, static_cast<const float*>(a.q) + (s.q_row * a.n_heads + hk * group) * d, r_first, n_rows, group, a.n_heads, d);
    const int len = seq_len(a, s);
    if (t < R) row_p[t] = t < n_rows ? query_pos(a, s, len, (r_first + t) / group) : -1;
    __syncthreads();
    int lo = 0x7FFFFFFF, hi = -1;                            // (positions below zero see nothing)
    for (int r = 0; r < n_rows; ++r)
        if (row_p[r] >= 0) { lo = min(lo, row_p[r]); hi = max(hi, row_p[r]); }
    const TileRange range = tile_range(a, len, lo, hi, kTile);
    const int per_split = (range.count + a.splits - 1) / a.splits;
    const int t0 = static_cast<int>(blockIdx.z) * per_split, t1 = min(range.count, t0 + per_split);
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * d;
    const float* const k = static_cast<const float*>(a.k) + s.kv_row * stride + static_cast<int64_t>(hk) * d;
    const float* const v = static_cast<const float*>(a.v) + s.kv_row * stride + static_cast<int64_t>(hk) * d;

    // The first tile from `it` on with a key that some row sees (t1: none), its positions in pos[buf], -1 for keys that no row sees (what they hold
    // is left out then); a barrier of the CTA at least once.
    const auto look = [&](int it) { return t < kTile && it < t1 ? key_pos(a, s, len, range.tile(it) * kTile + t) : -1; };
    const auto find = [&](int it, int c, int buf) {
        while (true) {
            bool seen = some_sees(lo, hi, c, a.window, a.n_sink);
            if (seen && a.q_pos) {                           // (queries may lie far apart)
                seen = false;
                for (int r = 0; r < n_rows && !seen; ++r) seen = sees(row_p[r], c, a.window, a.n_sink);
            }
            if (t < kTile) pos[buf][t] = seen ? c : -1;
            if (__syncthreads_or(seen)) return it;
            if (it >= t1) return t1;
            c = look(++it);
        }
    };
    const int rq = t / 16 * RT, kq = t % 16;
    const bool works = t / 32 * 2 * RT < n_rows;             // (a warp without rows only copies)
    float o[RT][NC][4] = {}, m[RT], l[RT];
    int p[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) { m[i] = -CUDART_INF_F; l[i] = 0.f; p[i] = row_p[rq + i]; }
    int buf = 0, it = find(t0, look(t0), 0);
    if (it < t1) copy_keys(ks, d + 4, k + range.tile(it) * static_cast<int64_t>(kTile) * stride, stride, d, pos[0]);
    copies_issued();
    while (it < t1) {
        const int c_next = look(it + 1);
        wait_copies<0>();
        __syncthreads();                                     // the keys are there; nobody reads the values any more
        copy_keys(vs, d, v + range.tile(it) * static_cast<int64_t>(kTile) * stride, stride, d, pos[buf]);
        copies_issued();
        float x[RT][kKeys], f[RT] = {};
        if (works) {
            dots<RT>(x, qs + rq * d, ks + kq * (d + 4), d);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float top = -CUDART_INF_F;
#pragma unroll
                for (int j = 0; j < kKeys; ++j) {
                    x[i][j] = sees(p[i], pos[buf][kq + 16 * j], a.window, a.n_sink) ? x[i][j] * a.scale_log2 : -CUDART_INF_F;
                    top = fmaxf(top, x[i][j]);
                }
#pragma unroll
                for (int w = 8; w >= 1; w /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                top = fmaxf(m[i], top);
                const float ref = top == -CUDART_INF_F ? 0.f : top;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < kKeys; ++j) {
                    x[i][j] = exp2f(x[i][j] - ref);
                    sum += x[i][j];
                    ps[(rq + i) * kPitch + kq + 16 * j] = x[i][j];
                }
                f[i] = exp2f(m[i] - ref);                        // 0 where there was nothing yet
                m[i] = top;
                l[i] = l[i] * f[i] + sum;                        // (this thread's keys)
            }
        }
        wait_copies<0>();
        const int next = find(it + 1, c_next, buf ^ 1);      // the values are there; nobody reads the keys any more
        if (next < t1) copy_keys(ks, d + 4, k + range.tile(next) * static_cast<int64_t>(kTile) * stride, stride, d, pos[buf ^ 1]);
        copies_issued();
        if (works) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] *= f[i];
            for (int j = 0; j < kTile; j += 4) {
                float w[RT][4];
#pragma unroll
                for (int i = 0; i < RT; ++i) *reinterpret_cast<float4*>(w[i]) = *reinterpret_cast<const float4*>(ps + (rq + i) * kPitch + j);
#pragma unroll
                for (int n = 0; n < NC; ++n) {
                    const int col = kq * 4 + 64 * n;
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) {
                        const float4 y = *reinterpret_cast<const float4*>(vs + (j + jj) * d + (col < d ? col : 0));
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            o[i][n][0] = fmaf(w[i][jj], y.x, o[i][n][0]);
                            o[i][n][1] = fmaf(w[i][jj], y.y, o[i][n][1]);
                            o[i][n][2] = fmaf(w[i][jj], y.z, o[i][n][2]);
                            o[i][n][3] = fmaf(w[i][jj], y.w, o[i][n][3]);
                        }
                    }
                }
            }
        }
        it = next;
        buf ^= 1;
    }
    wait_copies<0>();
    const bool whole = a.splits == 1;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int w = 8; w >= 1; w /= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        const int rr = r_first + rq + i, query = rr / group, h = hk * group + rr % group;
        if (rq + i >= n_rows) continue;
        const float f = whole ? (l[i] > 0.f ? 1.f / l[i] : 0.f) : 1.f;
        const int64_t part = (s.part0 + static_cast<int64_t>(blockIdx.z) * s.n_q + query) * a.n_heads + h;
        float* const out = whole ? static_cast<float*>(a.out) + ((s.q_row + query) * a.n_heads + h) * d : a.part_o + part * d;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int col = kq * 4 + 64 * n;
            if (col < d) *reinterpret_cast<float4*>(out + col) = make_float4(o[i][n][0] * f, o[i][n][1] * f, o[i][n][2] * f, o[i][n][3] * f);
        }
        if (kq != 0) continue;
        if (whole) {
            const float z = l[i] > 0.f ? m[i] + log2f(l[i]) : -CUDART_INF_F;
            if (a.lse) a.lse[(s.q_row + query) * a.n_heads + h] = z * 0.69314718055994531f;      // ln 2
            if (a.mass) a.lse2[static_cast<int64_t>(s.qp0 + query) * a.n_heads + h] = z;
        } else {
            a.part_ml[part] = make_float2(m[i], l[i]);
        }
    }
}

size_t mass_smem(int d) { return sizeof(float) * (kTile * (d + 4) + 2u * 32 * d); }

// One CTA: 64 cached rows of a sequence, one key head; its queries in blocks of 32 rows, every gridDim.z-th in order, the next block copied
// while one is worked on.
__global__ void __launch_bounds__(kThreads) mass_fma_kernel(const __grid_constant__ AttArgs a)
{
    constexpr int RT = 4, R = 8 * RT;
    extern __shared__ __align__(16) float sm[];
    __shared__ int row_p[3][R], pos[kTile];
    __shared__ float row_z[3][R], sums[8][kTile];
    const int d = a.head_dim, t = threadIdx.x;
    float* const ks = sm;
    float* const qs = ks + kTile * (d + 4);
    pdl_wait();
    pdl_trigger();
    int b = 0, tile = blockIdx.x;
    while (b + 1 < a.n_seq && tile >= (a.s[b].n_kv + kTile - 1) / kTile) tile -= (a.s[b++].n_kv + kTile - 1) / kTile;
    const AttSeq& s = a.s[b];
    const int hk = blockIdx.y, group = a.n_heads / a.kv_heads;
    const int len = seq_len(a, s), j0 = tile * kTile, total = s.n_q * group, step = static_cast<int>(gridDim.z) * R;
    const int64_t stride = static_cast<int64_t>(a.kv_heads) * d;
    if (t < kTile) pos[t] = key_pos(a, s, len, j0 + t);
    __syncthreads();
    int c_lo = 0x7FFFFFFF, c_hi = -1;
    for (int j = 0; j < kTile; ++j)
        if (pos[j] >= 0) { c_lo = min(c_lo, pos[j]); c_hi = max(c_hi, pos[j]); }
    copy_keys(ks, d + 4, static_cast<const float*>(a.k) + (s.kv_row + j0) * stride + static_cast<int64_t>(hk) * d, stride, d, pos);

    const float* const q = static_cast<const float*>(a.q) + (s.q_row * a.n_heads + hk * group) * d;
    // The first block of rows from r0 on that may see one of the keys (total: none), its positions and logarithms in buffer `at`.
    const auto find = [&](int r0, int at) {
        for (; r0 < total; r0 += step) {
            int p = -1;
            if (t < R) {
                const int rr = r0 + t;
                if (rr < total) p = query_pos(a, s, len, rr / group);
                row_p[at][t] = p;
                row_z[at][t] = rr < total ? a.lse2[static_cast<int64_t>(s.qp0 + rr / group) * a.n_heads + hk * group + rr % group] : 0.f;
            }
            if (__syncthreads_or(p >= c_lo && (c_lo < a.n_sink || p < c_hi || p - c_hi < a.window))) return r0;
        }
        return total;
    };
    const int rq = t / 16 * RT, kq = t % 16;
    float sum[kKeys] = {};
    int r0 = c_hi < 0 ? total : find(static_cast<int>(blockIdx.z) * R, 0);
    if (r0 < total) copy_queries<R>(qs, q, r0, min(R, total - r0), group, a.n_heads, d);
    copies_issued();
    for (int n = 0; r0 < total; ++n) {
        // (three buffers of positions: a thread may still be with the last block while another looks for the next)
        const int at = n % 3, next = find(r0 + step, (n + 1) % 3);
        __syncthreads();                                     // nobody is with the last block any more
        if (next < total) copy_queries<R>(qs + (n + 1) % 2 * R * d, q, next, min(R, total - next), group, a.n_heads, d);
        copies_issued();
        wait_copies<1>();
        __syncthreads();                                     // the keys and this block are there
        float x[RT][kKeys];
        dots<RT>(x, qs + n % 2 * R * d + rq * d, ks + kq * (d + 4), d);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int p = row_p[at][rq + i];
            const float z = row_z[at][rq + i];
#pragma unroll
            for (int j = 0; j < kKeys; ++j) sum[j] += sees(p, pos[kq + 16 * j], a.window, a.n_sink) ? exp2f(x[i][j] * a.scale_log2 - z) : 0.f;
        }
        r0 = next;
    }
    wait_copies<0>();
#pragma unroll
    for (int j = 0; j < kKeys; ++j) sums[t / 16][kq + 16 * j] = sum[j];
    __syncthreads();
    if (t < kTile && j0 + t < s.n_kv) {
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) all += sums[w][t];
        a.part_mass[(static_cast<int64_t>(hk) * gridDim.z + blockIdx.z) * a.total_kv + s.kvp0 + j0 + t] = all;
    }
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

template <int RT, int NC>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    return launch(setup, attend_fma_kernel<RT, NC>, dim3(static_cast<unsigned>(a.n_blocks), static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits)),
                  attend_smem(8 * RT, a.head_dim), a, stream);
}
template <int RT>
cudaError_t attend(const AttArgs& a, cudaStream_t stream)
{
    switch ((a.head_dim + 63) / 64) {
    case 1: return attend<RT, 1>(a, stream);
    case 2: return attend<RT, 2>(a, stream);
    case 3: return attend<RT, 3>(a, stream);
    default: return attend<RT, 4>(a, stream);                // (256 at most: the context's rule)
    }
}

}  // namespace

cudaError_t launch_attend_fma(const AttArgs& a, int rows, cudaStream_t stream) { return rows == 8 ? attend<1>(a, stream) : attend<4>(a, stream); }

cudaError_t launch_mass_fma(const AttArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    int64_t tiles = 0;
    for (int b = 0; b < a.n_seq; ++b) tiles += (a.s[b].n_kv + kTile - 1) / kTile;
    if (tiles == 0) return cudaSuccess;
    return launch(setup, mass_fma_kernel, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.mass_parts / a.kv_heads)), mass_smem(a.head_dim), a, stream);
}

}  // namespace mvla
