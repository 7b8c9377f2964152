// Rows of keys and values into pages, quantised on the way, and out of them again.
//
//   scale = the least 2^e with max |x| <= M 2^e;  code = x / scale rounded to the nearest       (M = 448 over a row of a head, or 6 over 32 elements)
//
// Bound by bytes.  Dividing by a power of two is exact, so that rounding to the code is the one rounding there is.  A lane has two pieces of eight neighbouring
// elements of a head (of bf16 16 bytes in one load or store, pieces of neighbouring lanes side by side), the lanes of a head are a power of two: the
// largest element crosses them by shuffles, of bf16 as pairs of 16-bit patterns, whose order is that of the numbers and leaves what is not
// finite on top.  A thread keeps its head and pieces from row to row; a CTA goes over blocks of rows, and where the next block's rows lie (their
// sequence, page and offsets) is looked up, a row by a thread, while one is worked on.
//
// B200: 12800 rows of 32 + 32 heads of 128 into bf16 pages 66 us (6.3 TB/s read and written), and out of them 65; 65537 rows of 8 + 8 heads to e2m1 70 us (4.8 TB/s; integer instructions 71 % of their
// pipe) and back 60; 131071 rows of 8 + 8 heads from e2m1 115 us (5.9 TB/s; reads of quantised bf16 rows spill 16 bytes or less at 64 registers, which four CTAs leave).  One piece to a lane and twice as many lanes: 149 us for the 65537 rows and back instead of 133 to 138.
#include "attend.cuh"
#include "page.cuh"

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = kRowThreads;
constexpr int kBlockRows = 32;               // of a CTA at a time, at most
constexpr int kPieces = 2;
constexpr int kWriteAhead = 2;               // rows of a thread on their way
template <int KIND> constexpr int kReadAhead = KIND == MVLA_PAGE_ROWS ? 2 : 4;
template <class T> constexpr int kCtas = sizeof(T) == 2 ? 4 : 3;      // that fit on a multiprocessor (by registers)

// Eight elements as they lie in memory; the largest magnitude; times 2^(byte - 127), as numbers; and back.
template <class T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void load(const void* p) { r = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(void* p) const { *static_cast<uint4*>(p) = r; }
    __device__ __forceinline__ void clear() { r = make_uint4(0, 0, 0, 0); }
    // of even and odd elements; over lanes and pieces by join; `top`: the bits of a 32-bit number
    __device__ __forceinline__ uint32_t largest() const { return join(join(r.x, r.y), join(r.z, r.w)); }
    static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b)
    {
        uint32_t c;
        asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));       // (the larger magnitude, of some sign; not a number, if one is none)
        return c;
    }
    static __device__ __forceinline__ uint32_t top(uint32_t a) { return join(a, a >> 16) << 16 & 0x7FFFFFFFu; }
    __device__ __forceinline__ void times(uint32_t byte, float (&x)[8]) const       // (what leaves the normal numbers is nothing among the codes)
    {
        const uint32_t ff = byte * 0x00800080u, w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), *reinterpret_cast<const __nv_bfloat162*>(&ff));
            const uint32_t y = *reinterpret_cast<const uint32_t*>(&h);
            x[2 * i] = __uint_as_float(y << 16);
            x[2 * i + 1] = __uint_as_float(y & 0xFFFF0000u);
        }
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
    __device__ __forceinline__ uint32_t largest() const
    {
        constexpr uint32_t m = 0x7FFFFFFFu;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) top = max(max(top, max(r[i].x & m, r[i].y & m)), max(r[i].z & m, r[i].w & m));
        return top;
    }
    static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t top(uint32_t a) { return a; }
    __device__ __forceinline__ void times(uint32_t byte, float (&x)[8]) const
    {
        const float f = __uint_as_float(byte << 23);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(r[i].x) * f;
            x[4 * i + 1] = __uint_as_float(r[i].y) * f;
            x[4 * i + 2] = __uint_as_float(r[i].z) * f;
            x[4 * i + 3] = __uint_as_float(r[i].w) * f;
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    }
};

// Eight numbers as codes (the first one lowest), rounded to the nearest; beyond the largest: the largest.
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8])
{
    uint2 w;
    asm("{\n\t.reg .b16 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 a, %3, %2;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 b, %5, %4;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 c, %7, %6;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 d, %9, %8;\n\t"
        "mov.b32 %0, {a, b};\n\t"
        "mov.b32 %1, {c, d};\n\t}"
        : "=r"(w.x), "=r"(w.y) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return w;
}
__device__ __forceinline__ uint32_t to_e2m1(const float (&x)[8])
{
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return w;
}

// Where a row of the batch lies; kZeros: it is none of the pool's, kNobodys: it is left alone.
constexpr int64_t kZeros = -1, kNobodys = -2;
constexpr int kTile = 64;
struct Place {
    int64_t k, v, at, scale;                 // bytes into k and v; of head 0's row into the pool's elements, or one of the above; and into its scales
};

template <int KIND, bool TILES, int WIDE>
__device__ __forceinline__ Place locate(const PageRowsArgs& a, int r)
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
    int64_t row;
    Place p;
    p.at = kZeros;
    if constexpr (TILES) {
        const TileRange range = counted_tiles(len, max(len - s.n_q, -1), max(len - 1, -1), kTile, a.window, a.n_sink);
        j = i / kTile < range.count ? range.tile(i / kTile) * kTile + i % kTile : -1;
        row = static_cast<int64_t>(r / kTile) * kTile * a.pool.kv_heads + r % kTile;
        p.at = kNobodys;
    } else {
        j = len - s.n_q + i;
        row = s.q_row + i;
    }
    p.k = row * a.k_stride * WIDE;
    p.v = row * a.v_stride * WIDE;
    if (j < 0 || j >= len) return p;
    const int page = page_of(a.pool, s.index, j);
    const int64_t at = page_row(a.pool, page, 0, j);
    p.at = page >= 0 ? at * page_row_bytes(KIND, a.pool.head_dim, WIDE) : kZeros;
    p.scale = at * page_row_scales(KIND, a.pool.head_dim);
    return p;
}

// Goes over this CTA's blocks of rows: work(places, rows) of each.
template <int KIND, bool TILES, int WIDE, class Work>
__device__ __forceinline__ void over_blocks(const PageRowsArgs& a, Place (*places)[kBlockRows], Work work)
{
    const int t = threadIdx.x, step = static_cast<int>(gridDim.x) * a.block_rows;
    int r0 = static_cast<int>(blockIdx.x) * a.block_rows, buf = 0;
    if (t < a.block_rows && r0 + t < a.total) places[0][t] = locate<KIND, TILES, WIDE>(a, r0 + t);
    __syncthreads();
    while (true) {
        const int64_t next = static_cast<int64_t>(r0) + step;
        const bool mine = t < a.block_rows && next + t < a.total;
        Place p;
        if (mine) p = locate<KIND, TILES, WIDE>(a, static_cast<int>(next) + t);
        work(places[buf], min(a.block_rows, a.total - r0));
        if (next >= a.total) break;
        if (mine) places[buf ^ 1][t] = p;
        __syncthreads();
        r0 = static_cast<int>(next);
        buf ^= 1;
    }
}

template <class T, int KIND, int LANES>
__global__ void __launch_bounds__(kThreads, kCtas<T>) page_write_kernel(const __grid_constant__ PageRowsArgs a)
{
    constexpr int kWide = sizeof(T);
    __shared__ Place places[2][kBlockRows];
    pdl_wait();
    pdl_trigger();
    const RowSlot s = row_slot(threadIdx.x, blockIdx.y, LANES, a.pool.kv_heads, a.k != nullptr, a.v != nullptr);
    const int d = a.pool.head_dim, row_bytes = page_row_bytes(KIND, d, kWide), groups = page_row_scales(KIND, d);
    const char* const src = static_cast<const char*>(s.values ? a.v : a.k) + s.head * (s.values ? a.v_head : a.k_head) * kWide;
    const int64_t head = static_cast<int64_t>(s.head) << a.pool.page_shift;
    uint8_t* const data = static_cast<uint8_t*>(s.values ? a.pool.v : a.pool.k) + head * row_bytes;
    uint8_t* const scales = KIND == MVLA_PAGE_ROWS ? nullptr : (s.values ? a.pool.v_scale : a.pool.k_scale) + head * groups;
    bool on[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) on[i] = s.on && (i * LANES + s.lane) * 8 < d;
    over_blocks<KIND, false, kWide>(a, places, [&](const Place* at, int n) {
        for (int b0 = 0; b0 < n; b0 += kWriteAhead * s.step) {    // (as often in every thread: shuffles)
            Eight<T> x[kWriteAhead][kPieces];
            int64_t to[kWriteAhead];
#pragma unroll
            for (int u = 0; u < kWriteAhead; ++u) {
                const int r = b0 + s.first + u * s.step;
                to[u] = r < n ? at[r].at : kZeros;
                const char* const from = src + (to[u] < 0 ? 0 : s.values ? at[r].v : at[r].k);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    x[u][i].clear();
                    if (to[u] >= 0 && on[i]) x[u][i].load(from + (i * LANES + s.lane) * 8 * kWide);
                }
            }
#pragma unroll
            for (int u = 0; u < kWriteAhead; ++u) {
                uint8_t* const dst = data + to[u];
                if constexpr (KIND == MVLA_PAGE_ROWS) {
#pragma unroll
                    for (int i = 0; i < kPieces; ++i)
                        if (to[u] >= 0 && on[i]) x[u][i].store(dst + (i * LANES + s.lane) * 8 * kWide);
                } else {
                    constexpr bool kE4m3 = KIND == MVLA_PAGE_E4M3;
                    uint32_t big[kPieces];
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) big[i] = x[u][i].largest();
                    if constexpr (kE4m3) big[0] = Eight<T>::join(big[0], big[1]);
#pragma unroll
                    for (int i = 0; i < (kE4m3 ? 1 : kPieces); ++i) {
#pragma unroll
                        for (int o = (kE4m3 ? LANES : kPageGroup / 8) / 2; o >= 1; o /= 2) big[i] = Eight<T>::join(big[i], __shfl_xor_sync(0xffffffffu, big[i], o));
                        big[i] = Eight<T>::top(big[i]);
                    }
                    if (to[u] < 0) continue;
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        if (!on[i]) continue;
                        const uint32_t top = big[kE4m3 ? 0 : i];
                        const bool finite = top < 0x7F800000u;
                        if (!finite) x[u][i].clear();
                        const uint32_t byte = finite ? scale_byte<KIND>(top) : 255u;
                        const int piece = i * LANES + s.lane;
                        float y[8];
                        x[u][i].times(finite ? 254u - byte : 0u, y);
                        if constexpr (kE4m3) {
                            *reinterpret_cast<uint2*>(dst + piece * 8) = to_e4m3(y);
                            if (piece == 0) scales[at[b0 + s.first + u * s.step].scale] = static_cast<uint8_t>(byte);
                        } else {
                            *reinterpret_cast<uint32_t*>(dst + piece * 4) = to_e2m1(y);
                            if (piece % (kPageGroup / 8) == 0) scales[at[b0 + s.first + u * s.step].scale + piece / (kPageGroup / 8)] = static_cast<uint8_t>(byte);
                        }
                    }
                }
            }
        }
    });
}

// TILES: for launch_page_tile and launch_page_fma; rows that no query sees are left out.
template <class T, int KIND, int LANES, bool TILES>
__global__ void __launch_bounds__(kThreads, kCtas<T>) page_read_kernel(const __grid_constant__ PageRowsArgs a)
{
    using Codes = std::conditional_t<KIND == MVLA_PAGE_ROWS, Eight<T>, std::conditional_t<KIND == MVLA_PAGE_E4M3, uint2, uint32_t>>;
    constexpr int kWide = sizeof(T), kAhead = kReadAhead<KIND>;
    __shared__ Place places[2][kBlockRows];
    pdl_wait();
    pdl_trigger();
    const RowSlot s = row_slot(threadIdx.x, blockIdx.y, LANES, a.pool.kv_heads, a.k != nullptr, a.v != nullptr);
    const int d = a.pool.head_dim, row_bytes = page_row_bytes(KIND, d, kWide), groups = page_row_scales(KIND, d);
    char* const dst = static_cast<char*>(s.values ? a.v : a.k) + s.head * (s.values ? a.v_head : a.k_head) * kWide;
    const int64_t head = static_cast<int64_t>(s.head) << a.pool.page_shift;
    const uint8_t* const data = static_cast<const uint8_t*>(s.values ? a.pool.v : a.pool.k) + head * row_bytes;
    const uint8_t* const scales = KIND == MVLA_PAGE_ROWS ? nullptr : (s.values ? a.pool.v_scale : a.pool.k_scale) + head * groups;
    bool on[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) on[i] = s.on && (i * LANES + s.lane) * 8 < d;
    over_blocks<KIND, TILES, kWide>(a, places, [&](const Place* at, int n) {
        for (int b0 = s.first; b0 < n; b0 += kAhead * s.step) {
            // (rows that are not there: codes of zero)
            Codes w[kAhead][kPieces];
            constexpr int kBytes = KIND == MVLA_PAGE_E2M1 ? kPieces : 1;
            uint32_t byte[kAhead][kBytes];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int r = b0 + u * s.step;
                const int64_t from = r < n ? at[r].at : kZeros;
                const uint8_t* const src = data + from;
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int piece = i * LANES + s.lane;
                    const bool there = from >= 0 && on[i];
                    if (i < kBytes) byte[u][i] = 127;
                    if constexpr (KIND == MVLA_PAGE_ROWS) {
                        w[u][i].clear();
                        if (there) w[u][i].load(src + piece * 8 * kWide);
                    } else {
                        w[u][i] = Codes{};
                        if (there) w[u][i] = *reinterpret_cast<const Codes*>(src + piece * (KIND == MVLA_PAGE_E4M3 ? 8 : 4));
                        if (i < kBytes && from >= 0) byte[u][i] = scales[at[r].scale + (KIND == MVLA_PAGE_E4M3 || !on[i] ? 0 : piece / (kPageGroup / 8))];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int r = b0 + u * s.step;
                if (r >= n || (TILES && at[r].at == kNobodys)) continue;
                char* const to = dst + (s.values ? at[r].v : at[r].k);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    Eight<T> y;
                    if constexpr (KIND == MVLA_PAGE_ROWS) {
                        y = w[u][i];
                    } else {
                        float x[8];
                        code_values(w[u][i], x);
                        const float scale = scale_value(byte[u][i < kBytes ? i : 0]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] *= scale;
                        y.set(x);
                    }
                    if (on[i]) y.store(to + (i * LANES + s.lane) * 8 * kWide);
                }
            }
        }
    });
}

int lanes_of(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

enum Way { kWrite, kRead, kTiles };
template <Way WAY, class T, int KIND, int LANES>
cudaError_t launch(PageRowsArgs& a, cudaStream_t stream)
{
    const int heads = (a.k ? a.pool.kv_heads : 0) + (a.v ? a.pool.kv_heads : 0);
    const int64_t slots = static_cast<int64_t>(heads) * LANES;
    const int columns = static_cast<int>((slots + kThreads - 1) / kThreads), step = slots >= kThreads ? 1 : static_cast<int>(kThreads / slots);
    // Blocks of as many rows as there can be while every multiprocessor has its CTAs, which go over the rest.  Plain copies: a CTA to every few rows
    // (12800 rows of 32 heads of 128 written: 68 us so, 80 with CTAs that stay; 12500 of 8 heads to e4m3 and back 34 us so, 31 with CTAs that stay).
    const int64_t ctas = kCtas<T> * static_cast<int64_t>(sm_count_of_current_device()), rows = (static_cast<int64_t>(a.total) * columns + ctas - 1) / ctas;
    const int64_t most = KIND == MVLA_PAGE_ROWS ? 2 * kWriteAhead * step : kBlockRows;
    a.block_rows = static_cast<int32_t>(std::min<int64_t>({std::max<int64_t>((rows + step - 1) / step * step, step), most, kBlockRows}));
    const int64_t blocks = (static_cast<int64_t>(a.total) + a.block_rows - 1) / a.block_rows, stay = KIND == MVLA_PAGE_ROWS ? blocks : std::max<int64_t>(1, ctas / columns);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min(blocks, stay)), static_cast<unsigned>(columns));
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
    case 4: return launch<WAY, T, KIND, 4>(a, stream);
    case 8: return launch<WAY, T, KIND, 8>(a, stream);
    default: return launch<WAY, T, KIND, 16>(a, stream);
    }
}
template <Way WAY, class T>
cudaError_t by_kind(int kind, PageRowsArgs& a, cudaStream_t stream)
{
    if constexpr (WAY != kTiles)                             // (tiles are made of quantised pages)
        if (kind == MVLA_PAGE_ROWS) return by_lanes<WAY, T, MVLA_PAGE_ROWS>(a, stream);
    return kind == MVLA_PAGE_E4M3 ? by_lanes<WAY, T, MVLA_PAGE_E4M3>(a, stream) : by_lanes<WAY, T, MVLA_PAGE_E2M1>(a, stream);
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
