// Rows of keys and values into pages, quantised on the way, and out of them again.
//
//   scale = the least 2^e with max |x| <= M 2^e;  code = x / scale rounded to the nearest       (M = 448 over a row of a head, or 6 over 32 elements)
//
// Bound by bytes.  Dividing by a power of two is exact, so that rounding to the code is the one rounding there is.  A lane has eight neighbouring
// elements of a head (16 bytes of bf16 in one load, the codes in one store), the lanes of a head are a power of two side by side: the
// largest element crosses them by shuffles, of bf16 as pairs of 16-bit patterns, whose order is that of the numbers and leaves what is not
// finite on top.  A CTA has a block of rows; where each of them lies is looked up once, by a thread, and a thread
// keeps its head and elements from row to row, four rows on their way at a time.
#include "attend.cuh"
#include "page.cuh"

#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlockRows = 64;
constexpr int kAhead = 4;                    // rows of a thread on their way

// Eight elements as they lie in memory; the largest magnitude's bits in 32 bits; and as numbers.
template <class T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void load(const void* p) { r = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(void* p) const { *static_cast<uint4*>(p) = r; }
    __device__ __forceinline__ void clear() { r = make_uint4(0, 0, 0, 0); }
    template <int LANES> __device__ __forceinline__ uint32_t largest() const
    {
        constexpr uint32_t m = 0x7FFF7FFFu;
        uint32_t top = __vmaxu2(__vmaxu2(r.x & m, r.y & m), __vmaxu2(r.z & m, r.w & m));
#pragma unroll
        for (int o = LANES / 2; o >= 1; o /= 2) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
        return max(top & 0xFFFFu, top >> 16) << 16;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Eight<float> {
    uint4 r[2];
    __device__ __forceinline__ void load(const void* p) { r[0] = static_cast<const uint4*>(p)[0]; r[1] = static_cast<const uint4*>(p)[1]; }
    __device__ __forceinline__ void store(void* p) const { static_cast<uint4*>(p)[0] = r[0]; static_cast<uint4*>(p)[1] = r[1]; }
    __device__ __forceinline__ void clear() { r[0] = r[1] = make_uint4(0, 0, 0, 0); }
    template <int LANES> __device__ __forceinline__ uint32_t largest() const
    {
        constexpr uint32_t m = 0x7FFFFFFFu;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) top = max(max(top, max(r[i].x & m, r[i].y & m)), max(r[i].z & m, r[i].w & m));
#pragma unroll
        for (int o = LANES / 2; o >= 1; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        return top;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(r[i].x);
            x[4 * i + 1] = __uint_as_float(r[i].y);
            x[4 * i + 2] = __uint_as_float(r[i].z);
            x[4 * i + 3] = __uint_as_float(r[i].w);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    }
};

constexpr int64_t kZeros = -1, kNobodys = -2;                // rows of the pool: none; and one that is left alone
constexpr int kTile = 64;

// Row r of the batch, packed: its row of k / v, and its row of head 0 in the pool, or one of the above.
template <bool TILES>
__device__ __forceinline__ void locate(const PageRowsArgs& a, int r, int64_t* row, int64_t* at)
{
    int b = 0, n = a.n_seq;
    while (n > 1) {                                          // the last sequence that begins at r or before
        const int half = n >> 1;
        if (a.s[b + half].row0 <= r) b += half;
        n -= half;
    }
    const PageSeq& s = a.s[b];
    const int len = a.kv_len ? min(max(a.kv_len[s.index], 0), s.n_kv) : s.n_kv, i = r - s.row0;
    int j;
    if constexpr (TILES) {
        const int lo = max(len - s.n_q, -1), hi = max(len - 1, -1);
        const TileRange range = counted_tiles(len, lo, hi, kTile, a.window, a.n_sink);
        j = i / kTile < range.count ? range.tile(i / kTile) * kTile + i % kTile : -1;
        *row = static_cast<int64_t>(r / kTile) * kTile * a.pool.kv_heads + r % kTile;
        *at = kNobodys;
        if (j < 0 || j >= len) return;
    } else {
        j = len - s.n_q + i;
        *row = s.q_row + i;
    }
    *at = kZeros;
    if (j < 0 || j >= len) return;
    const int page = page_of(a.pool, s.index, j);
    if (page >= 0) *at = page_row(a.pool, page, 0, j);
}

// A thread's place in the rows of its CTA: which tensor, head and elements it has, and in which rows.
struct Slot {
    bool values, on;
    int head, sub, first, step;
};
template <int LANES>
__device__ __forceinline__ Slot slot_of(const PageRowsArgs& a)
{
    const int heads = (a.k ? a.pool.kv_heads : 0) + (a.v ? a.pool.kv_heads : 0), slots = heads * LANES;
    const int t = threadIdx.x;
    Slot s;
    int u;
    if (slots >= kThreads) {
        u = static_cast<int>(blockIdx.y) * kThreads + t;
        s.first = 0;
        s.step = 1;
    } else {
        s.step = kThreads / slots;
        s.first = t / slots;
        u = t - s.first * slots;
        if (s.first >= s.step) u = slots;
    }
    s.sub = u % LANES;
    const int h = u / LANES;
    s.values = !a.k || h >= a.pool.kv_heads;
    s.head = s.values && a.k ? h - a.pool.kv_heads : h;
    s.on = u < slots && s.sub * 8 < a.pool.head_dim;
    return s;
}

template <class T, int KIND, int LANES>
__global__ void __launch_bounds__(kThreads) page_write_kernel(const __grid_constant__ PageRowsArgs a)
{
    __shared__ int64_t rows[kMaxBlockRows], ats[kMaxBlockRows];
    pdl_wait();
    pdl_trigger();
    const int r0 = static_cast<int>(blockIdx.x) * a.block_rows, n = min(a.block_rows, a.total - r0);
    if (static_cast<int>(threadIdx.x) < n) locate<false>(a, r0 + threadIdx.x, &rows[threadIdx.x], &ats[threadIdx.x]);
    __syncthreads();
    const Slot s = slot_of<LANES>(a);
    const int d = a.pool.head_dim, c = s.sub * 8;
    const char* const src = static_cast<const char*>(s.values ? a.v : a.k) + (s.head * (s.values ? a.v_head : a.k_head) + c) * static_cast<int64_t>(sizeof(T));
    const int64_t stride = (s.values ? a.v_stride : a.k_stride) * static_cast<int64_t>(sizeof(T));
    uint8_t* const data = static_cast<uint8_t*>(s.values ? a.pool.v : a.pool.k);
    uint8_t* const scales = s.values ? a.pool.v_scale : a.pool.k_scale;
    const int64_t head = static_cast<int64_t>(s.head) << a.pool.page_shift;
    for (int b0 = 0; b0 < n; b0 += kAhead * s.step) {        // (as often in every thread: shuffles)
        Eight<T> x[kAhead];
        int64_t at[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = b0 + s.first + u * s.step;
            at[u] = s.on && r < n ? ats[r] : -1;
            x[u].clear();
            if (at[u] >= 0) x[u].load(src + rows[r] * stride);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t to = at[u] + head;
            if constexpr (KIND == MVLA_PAGE_ROWS) {
                if (at[u] >= 0) x[u].store(data + (to * d + c) * static_cast<int64_t>(sizeof(T)));
            } else {
                constexpr bool kE4m3 = KIND == MVLA_PAGE_E4M3;
                const uint32_t big = x[u].template largest<kE4m3 ? LANES : kPageGroup / 8>();
                if (at[u] < 0) continue;
                const bool finite = big < 0x7F800000u;
                const int e = scale_exponent<KIND>(big);
                const float per = finite ? two_to(-e) : 0.f;
                float y[8];
                x[u].get(y);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = finite ? y[i] * per : 0.f;
                const uint8_t byte = finite ? static_cast<uint8_t>(e + 127) : 255;
                if constexpr (kE4m3) {
                    uint2 w = {0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(y[2 * i], y[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
                        (i < 2 ? w.x : w.y) |= two << (16 * (i & 1));
                    }
                    *reinterpret_cast<uint2*>(data + to * d + c) = w;
                    if (s.sub == 0) scales[to] = byte;
                } else {
                    uint32_t w = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w |= static_cast<uint32_t>(__nv_cvt_float2_to_fp4x2(make_float2(y[2 * i], y[2 * i + 1]), __NV_E2M1, cudaRoundNearest)) << (8 * i);
                    *reinterpret_cast<uint32_t*>(data + (to * d + c) / 2) = w;
                    if (s.sub % (kPageGroup / 8) == 0) scales[to * (d / kPageGroup) + c / kPageGroup] = byte;
                }
            }
        }
    }
}

// TILES: for launch_page_tile; rows that no query sees are left out.
template <class T, int KIND, int LANES, bool TILES>
__global__ void __launch_bounds__(kThreads) page_read_kernel(const __grid_constant__ PageRowsArgs a)
{
    using Codes = std::conditional_t<KIND == MVLA_PAGE_ROWS, Eight<T>, std::conditional_t<KIND == MVLA_PAGE_E4M3, uint2, uint32_t>>;
    __shared__ int64_t rows[kMaxBlockRows], ats[kMaxBlockRows];
    pdl_wait();
    pdl_trigger();
    const int r0 = static_cast<int>(blockIdx.x) * a.block_rows, n = min(a.block_rows, a.total - r0);
    if (static_cast<int>(threadIdx.x) < n) locate<TILES>(a, r0 + threadIdx.x, &rows[threadIdx.x], &ats[threadIdx.x]);
    __syncthreads();
    const Slot s = slot_of<LANES>(a);
    if (!s.on) return;
    const int d = a.pool.head_dim, c = s.sub * 8;
    char* const dst = static_cast<char*>(s.values ? a.v : a.k) + (s.head * (s.values ? a.v_head : a.k_head) + c) * static_cast<int64_t>(sizeof(T));
    const int64_t stride = (s.values ? a.v_stride : a.k_stride) * static_cast<int64_t>(sizeof(T));
    const uint8_t* const data = static_cast<const uint8_t*>(s.values ? a.pool.v : a.pool.k);
    const uint8_t* const scales = s.values ? a.pool.v_scale : a.pool.k_scale;
    const int64_t head = static_cast<int64_t>(s.head) << a.pool.page_shift;
    for (int b0 = s.first; b0 < n; b0 += kAhead * s.step) {
        Codes w[kAhead];
        uint32_t byte[kAhead];
        bool there[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = b0 + u * s.step;
            const int64_t from = r < n ? ats[r] : -1, at = from + head;
            there[u] = from >= 0;
            if (!there[u]) continue;
            if constexpr (KIND == MVLA_PAGE_ROWS) {
                w[u].load(data + (at * d + c) * static_cast<int64_t>(sizeof(T)));
            } else {
                w[u] = *reinterpret_cast<const Codes*>(data + (KIND == MVLA_PAGE_E4M3 ? at * d + c : (at * d + c) / 2));
                byte[u] = scales[KIND == MVLA_PAGE_E4M3 ? at : at * (d / kPageGroup) + c / kPageGroup];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = b0 + u * s.step;
            if (r >= n) break;
            if (TILES && ats[r] == kNobodys) continue;
            Eight<T> y;
            y.clear();
            if (there[u]) {
                if constexpr (KIND == MVLA_PAGE_ROWS) {
                    y = w[u];
                } else {
                    float x[8];
                    code_values(w[u], x);
                    const float scale = scale_value(byte[u]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= scale;
                    y.set(x);
                }
            }
            y.store(dst + rows[r] * stride);
        }
    }
}

int lanes_of(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

enum Way { kWrite, kRead, kTiles };
template <Way WAY, class T, int KIND, int LANES>
cudaError_t launch(PageRowsArgs& a, cudaStream_t stream)
{
    const int heads = (a.k ? a.pool.kv_heads : 0) + (a.v ? a.pool.kv_heads : 0);
    const int64_t slots = static_cast<int64_t>(heads) * LANES;
    const int columns = static_cast<int>((slots + kThreads - 1) / kThreads), step = slots >= kThreads ? 1 : static_cast<int>(kThreads / slots);
    // rows of a CTA: what its threads have on their way at a time, up to four times as many where that still fills the device
    const int64_t pass = static_cast<int64_t>(step) * kAhead, ctas = (a.total + pass - 1) / pass * columns, fill = 8 * static_cast<int64_t>(sm_count_of_current_device());
    int64_t block = ctas >= 4 * fill ? 4 * pass : ctas >= 2 * fill ? 2 * pass : pass;
    if (ctas < fill) block = step;                           // few rows: each its own CTA, where that helps
    a.block_rows = static_cast<int32_t>(std::min<int64_t>(block, kMaxBlockRows));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((a.total + a.block_rows - 1) / a.block_rows), static_cast<unsigned>(columns));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if constexpr (WAY == kWrite) return cudaLaunchKernelEx(&cfg, page_write_kernel<T, KIND, LANES>, a);
    else return cudaLaunchKernelEx(&cfg, page_read_kernel<T, KIND, LANES, WAY == kTiles>, a);
}
template <Way WAY, class T, int KIND>
cudaError_t by_lanes(PageRowsArgs& a, cudaStream_t stream)
{
    switch (lanes_of(a.pool.head_dim)) {
    case 8: return launch<WAY, T, KIND, 8>(a, stream);
    case 16: return launch<WAY, T, KIND, 16>(a, stream);
    default: return launch<WAY, T, KIND, 32>(a, stream);
    }
}
template <Way WAY, class T>
cudaError_t by_kind(int kind, PageRowsArgs& a, cudaStream_t stream)
{
    switch (kind) {
    case MVLA_PAGE_ROWS: return by_lanes<WAY, T, MVLA_PAGE_ROWS>(a, stream);
    case MVLA_PAGE_E4M3: return by_lanes<WAY, T, MVLA_PAGE_E4M3>(a, stream);
    default: return by_lanes<WAY, T, MVLA_PAGE_E2M1>(a, stream);
    }
}

}  // namespace

cudaError_t launch_page_write(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream)
{
    return hidden_dtype == MVLA_DTYPE_FP32 ? by_kind<kWrite, float>(kind, a, stream) : by_kind<kWrite, __nv_bfloat16>(kind, a, stream);
}
cudaError_t launch_page_read(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream)
{
    return hidden_dtype == MVLA_DTYPE_FP32 ? by_kind<kRead, float>(kind, a, stream) : by_kind<kRead, __nv_bfloat16>(kind, a, stream);
}
cudaError_t launch_page_tiles(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream)
{
    return hidden_dtype == MVLA_DTYPE_FP32 ? by_kind<kTiles, float>(kind, a, stream) : by_kind<kTiles, __nv_bfloat16>(kind, a, stream);
}

}  // namespace mvla
