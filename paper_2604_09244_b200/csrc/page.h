// Launchers of the calls on a cache in pages (page_*.cu) and what they are given.
#pragma once

#include "page_plan.h"
#include "serve.h"

namespace mvla {

struct PagePool {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t* table;
    int64_t table_stride;
    int64_t n_pages;
    int32_t page_shift;                      // page_rows = 1 << page_shift
    int32_t kv_heads, head_dim;
};

// ---- rows into pages and out of them

struct PageSeq {
    int64_t q_row;
    int32_t n_q, n_kv;
    int32_t row0;                            // its first row among those of the batch, packed
    int32_t index;                           // its place in the caller's batch
};
struct PageRowsArgs {
    PagePool pool;
    const int32_t* kv_len;
    void *k, *v;                             // each null: left alone
    int64_t k_stride, v_stride;
    int32_t n_seq, total;                    // rows of the batch
    int32_t block_rows;                      // rows of a CTA
    int64_t k_head, v_head;                  // elements from one head of a row to the next
    // launch_page_tiles: the rows of the tiles of 64 that a sequence's queries see, tile after tile, of every tile head after head.  Of s: n_q, n_kv, and as
    // row0 64 times the sequence's first tile
    int32_t window, n_sink;
    PageSeq s[kMaxBatch];
};
cudaError_t launch_page_write(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream);
cudaError_t launch_page_read(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream);
cudaError_t launch_page_tiles(int hidden_dtype, int kind, PageRowsArgs& a, cudaStream_t stream);

// ---- attention

// Single tokens (launch_attend_token's), over pages; q and out bf16.  Behind it: launch_attend_finish.
cudaError_t launch_page_token(int kind, const AttArgs& a, const PagePool& pool, int rows, cudaStream_t stream);

// Blocks of `row_tiles` (1, or 2 for heads of up to 128 elements) tiles of 128 query rows over quantised pages, unpacked on the way; q and out bf16.  Behind it: launch_attend_join.
cudaError_t launch_page_decode(int kind, int row_tiles, const AttArgs& a, const PagePool& pool, cudaStream_t stream);

// fp32, by FMAs, in blocks of 8 query rows.  Behind it: launch_attend_join.
cudaError_t launch_page_fma(const AttArgs& a, cudaStream_t stream);

}  // namespace mvla
