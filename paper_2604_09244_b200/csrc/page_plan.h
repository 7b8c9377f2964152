// Sizes of a cache in pages that plans and kernels go by.
#pragma once

#include "mvla_prune.h"

#ifdef __CUDACC__
#define MVLA_BOTH __host__ __device__
#else
#define MVLA_BOTH
#endif

namespace mvla {

constexpr int kPageGroup = 32;               // elements that share a scale in e2m1 pages
// Exponents of the scales: from 2^-117 on every element that the codes can stand for is a normal number of 32 bits and of bf16; up to 2^119 (e4m3) and 2^125
// (e2m1) it is a finite one.
constexpr int kScaleLeast = -117, kScaleMostE4m3 = 119, kScaleMostE2m1 = 125;

// Bytes of a cached row of one head, and of its scales.
MVLA_BOTH constexpr int page_row_bytes(int kind, int d, int wide) { return kind == MVLA_PAGE_ROWS ? d * wide : kind == MVLA_PAGE_E4M3 ? d : d / 2; }
MVLA_BOTH constexpr int page_row_scales(int kind, int d) { return kind == MVLA_PAGE_ROWS ? 0 : kind == MVLA_PAGE_E4M3 ? 1 : d / kPageGroup; }

// Rows into pages and out (page_rows.cu): a thread's place in the rows of its CTA, which tensor, head and lane of the head it has, and in which rows.
constexpr int kRowThreads = 256;
struct RowSlot {
    bool values, on;
    int head, lane, first, step;
};
MVLA_BOTH constexpr RowSlot row_slot(int thread, int column, int lanes, int kv_heads, bool keys, bool values)
{
    const int heads = (keys ? kv_heads : 0) + (values ? kv_heads : 0), slots = heads * lanes;
    int u = column * kRowThreads + thread, first = 0, step = 1;
    if (slots < kRowThreads) {
        step = kRowThreads / slots;
        first = thread / slots;
        u = first < step ? thread - first * slots : slots;
    }
    const bool on = u < slots;
    const int h = on ? u / lanes : 0;                        // (the surplus threads copy nothing; what they form addresses of, and the scales that they read, are there all the same)
    return {!keys || h >= kv_heads, on, keys && h >= kv_heads ? h - kv_heads : h, u % lanes, first, step};
}

// Single tokens (page_token.cu): subtiles of 16 keys in a warp's tile, bytes of a tile in shared memory (in whole groups of 64 columns of the values),
// tiles of a warp, and the CTAs that fit on a multiprocessor.
constexpr int kPageTokenStages = 2;
MVLA_BOTH constexpr int page_token_sub(int kind, int pieces_of_32) { return pieces_of_32 <= 2 || (kind != MVLA_PAGE_ROWS && pieces_of_32 <= 4) ? 2 : 1; }
MVLA_BOTH constexpr int page_token_tile(int kind, int pieces_of_32)
{
    const int run = kind == MVLA_PAGE_ROWS ? 16 : kind == MVLA_PAGE_E4M3 ? 8 : 4, scales = kind == MVLA_PAGE_ROWS ? 0 : kind == MVLA_PAGE_E4M3 ? 1 : pieces_of_32;
    return page_token_sub(kind, pieces_of_32) * ((2 * pieces_of_32 + 4 * ((pieces_of_32 + 1) / 2)) * 32 * run + 32 * scales);
}
// (`groups`: of eight query rows)
MVLA_BOTH constexpr int page_token_ctas(int kind, int pieces_of_32, int groups)
{
    // queries, factors of the scales, and what the system takes; registers: four CTAs leave 128 to a thread, three 168, two 255
    const int fixed = 512 * groups * pieces_of_32 + (kind == MVLA_PAGE_E2M1 ? 256 * page_token_sub(kind, pieces_of_32) * pieces_of_32 : 0) + 3 * 1024;
    const int n = 227 * 1024 / (4 * kPageTokenStages * page_token_tile(kind, pieces_of_32) + fixed), most = groups == 1 ? (pieces_of_32 <= 6 ? 4 : 3) : pieces_of_32 <= 2 ? 3 : 2;
    return n > most ? most : n < 1 ? 1 : n;
}

// Few fp32 rows (page_fma.cu): warps of a CTA, and the CTAs that fit on a multiprocessor.
MVLA_BOTH constexpr int page_fma_warps(int pieces_of_32) { return pieces_of_32 <= 2 ? 8 : 4; }
MVLA_BOTH constexpr int page_fma_ctas(int pieces_of_32) { return pieces_of_32 <= 2 ? 2 : pieces_of_32 <= 4 ? 3 : pieces_of_32 <= 6 ? 2 : 1; }

}  // namespace mvla
