// Device side of a cache in pages that its kernels share: where a cached row lies, and what codes and scales stand for.
#pragma once

#include "device_utils.cuh"
#include "page.h"

#include <cuda_fp16.h>

namespace mvla {

// Page of cached row j of the batch's sequence `index`, -1 where it is none of the pool's.
__device__ __forceinline__ int page_of(const PagePool& p, int index, int j)
{
    const int page = p.table[index * p.table_stride + (j >> p.page_shift)];
    return page >= 0 && page < p.n_pages ? page : -1;
}
// Row of head h's rows [n_pages, kv_heads, page_rows] that row j of a sequence is, on its page.
__device__ __forceinline__ int64_t page_row(const PagePool& p, int page, int h, int j)
{
    return ((static_cast<int64_t>(page) * p.kv_heads + h) << p.page_shift) + (j & ((1 << p.page_shift) - 1));
}

// The byte of the least scale 2^e, e not below kScaleLeast, with |x| <= M 2^e for the largest |x| of a group, whose bits in 32 bits these are (finite): M = 448 = 1.75
// 2^8 or 6 = 1.5 2^2, and a larger fraction than M's carries into the exponent.
template <int KIND>
__device__ __forceinline__ uint32_t scale_byte(uint32_t big)
{
    constexpr bool kE4m3 = KIND == MVLA_PAGE_E4M3;
    const int e = static_cast<int>((big + (kE4m3 ? 0x1FFFFFu : 0x3FFFFFu)) >> 23) - (kE4m3 ? 8 : 2);
    return static_cast<uint32_t>(min(max(e, kScaleLeast + 127), (kE4m3 ? kScaleMostE4m3 : kScaleMostE2m1) + 127));
}
// 2^e for a normal number's e.
__device__ __forceinline__ float two_to(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// What a scale's byte stands for.
__device__ __forceinline__ float scale_value(uint32_t byte) { return byte == 255u ? CUDART_NAN_F : byte == 0u ? 0x1p-127f : __uint_as_float(byte << 23); }

// The codes of a register as fp16 pairs: one instruction to a pair.  (The conversions of the headers take a pair as a number of its own and hand back two halves: 7
// cycles of a warp to a pair of e4m3, 10 to one of e2m1, instead of 2.)
__device__ __forceinline__ void from_e4m3(uint32_t four, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(four));
}
__device__ __forceinline__ void from_e2m1(uint32_t eight, uint32_t (&x)[4])
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(eight));
}
// Eight codes as numbers.
__device__ __forceinline__ void code_values(const uint32_t (&h)[4], float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void code_values(uint2 codes, float (&x)[8])
{
    uint32_t h[4];
    from_e4m3(codes.x, h[0], h[1]);
    from_e4m3(codes.y, h[2], h[3]);
    code_values(h, x);
}
__device__ __forceinline__ void code_values(uint32_t codes, float (&x)[8])
{
    uint32_t h[4];
    from_e2m1(codes, h);
    code_values(h, x);
}

}  // namespace mvla
