// Launchers of the calls around the prune point (rope.cu, attend_*.cu, evict.cu) and what they are given.
#pragma once

#include "api_util.h"

namespace mvla {

struct RopeJob {
    const void *q, *k, *v, *q_weight, *k_weight;
    int64_t n_rows, q_stride, k_stride, v_stride, kv_rows;
    const int32_t* pos;
    const double* inv_freq;
    const int32_t* out_rows;
    void *q_out, *k_out, *v_out;
    int32_t n_heads, kv_heads, head_dim, rot_dim;
    float eps;
    bool norm, interleaved;
};
// dtype: MVLA_DTYPE_* of the outputs (fp32 from fp32 inputs, bf16 and e4m3 from bf16).
cudaError_t launch_qk_norm_rope(int dtype, const RopeJob& job, cudaStream_t stream);

// ---- windowed attention

// One sequence of a launch.
struct AttSeq {
    int64_t q_row, kv_row;
    int32_t n_q, n_kv;
    int32_t blk0;                // first of its blocks of query rows in the launch (a block: rows of one key head)
    int32_t qp0, kvp0;           // its first query / cached row among those of the batch, packed
    int32_t tile0;               // first of its tiles of 128 cached rows
    int32_t parts;               // parts that its visible keys are cut into
    int64_t part0;               // first of its queries among the parts' results: [parts][n_q] of them
    int64_t logit0;              // first of its scores (single tokens with mass): [n_q][n_heads][n_kv]
    int32_t qm_row, km_row;      // where its queries and cached rows begin in the tensor maps (kernels by tiles)
    int32_t index;               // its place in the caller's batch (kv_len)
};
struct AttArgs {
    const void *q, *k, *v;
    void* out;
    float *lse, *mass;
    const int32_t *q_pos, *kv_pos, *kv_len;
    int32_t n_heads, kv_heads, head_dim, window, n_sink;
    float scale_log2;            // scale of the dot products, in powers of two
    int32_t n_seq, n_blocks, total_q, total_kv;
    int32_t splits;              // the most parts that the visible keys of a sequence are cut into
    // workspace
    float* part_o;               // [parts' queries][n_heads][head_dim] sums against the part's own reference      (splits > 1)
    float2* part_ml;             // [parts' queries][n_heads] (reference, sum of exponentials), powers of two
    float* lse2;                 // [total_q][n_heads] logarithm to base 2 of the sum of exponentials          (with mass)
    float* part_mass;            // [mass_parts][total_kv]                                                     (with mass)
    int32_t mass_parts;
    int32_t skip_whole;          // sequences of one part have written their output themselves (single tokens)
    float* logits;               // scores in powers of two, -infinity where a row is not seen                (single tokens with mass)
    int32_t pack;                // heads of a group side by side in a tile of rows (kernels by tiles)
    int* status;                 // word that receives MVLA_ERR_TIMEOUT when a bounded wait gives up
    // pages (launch_page_tile, launch_page_fma)
    const int32_t* table;        // null: the tiles that a sequence's queries see lie one after another, from tile km_row on
    int64_t table_stride;
    int32_t n_pages, page_shift; // page_rows = 1 << page_shift
    int32_t cluster;             // CTAs to a cluster (launch_page_token, launch_page_tile, launch_page_decode): a sequence's parts are its clusters
    AttSeq s[kMaxBatch];
};

// fp32, by FMAs: any shape, in blocks of `rows` (8 or 32) query rows.
cudaError_t launch_attend_fma(const AttArgs& a, int rows, cudaStream_t stream);
// The weights of every cached row over the queries of its sequence, by key head, into part_mass (by FMAs in 32 bits).
cudaError_t launch_mass_fma(const AttArgs& a, cudaStream_t stream);
// bf16 (f16: what launch_widen made) by tiles of 128 rows on the tensor cores; at most kMaxTiles tiles of keys to a split.
struct AttMaps {
    CUtensorMap q, k, v;
};
// `tokens`: bf16, and some sequence counts as single tokens (kTokenRows).
cudaError_t launch_attend_tile(bool f16, bool tokens, const AttArgs& a, const AttMaps& maps, cudaStream_t stream);
// The same over pages: maps.k and maps.v of (head_dim, rows of a page, pages x key heads), boxes of as many rows as a page has, 64 at most.
cudaError_t launch_page_tile(bool tokens, const AttArgs& a, const AttMaps& maps, cudaStream_t stream);
// The weights as above, by tiles of 128 keys.  (mass_parts: packs of heads, times runs of kMaxTiles tiles of queries)
cudaError_t launch_attend_weights(bool f16, const AttArgs& a, const AttMaps& maps, cudaStream_t stream);
// The sequences' e4m3 rows as packed fp16 rows.
cudaError_t launch_widen(const AttArgs& a, void* wide_q, void* wide_k, void* wide_v, cudaStream_t stream);
// bf16 / e4m3, at most 16 query rows (queries x heads of a group) to a sequence and key head; `rows`: the most there are.  A block: a
// part of a sequence's keys.
cudaError_t launch_attend_token(int dtype, const AttArgs& a, int rows, cudaStream_t stream);
// Behind it: the parts joined, and mass += the weights that the kept scores stand for.
cudaError_t launch_attend_finish(const AttArgs& a, cudaStream_t stream);
// part_o / part_ml -> out, lse, lse2.
cudaError_t launch_attend_join(int dtype, bool by_ctas, const AttArgs& a, cudaStream_t stream);
// mass += part_mass over its parts.
cudaError_t launch_mass_add(const AttArgs& a, cudaStream_t stream);

// What the kernels of a checked call are given.
void fill_attention(AttArgs& k, const CtxView& v, int32_t batch, const mvla_seq* seqs, const mvla_attention* a, const AttendPlan& plan);

// ---- eviction by accumulated weight

struct EvictSeq {
    int64_t kv_row;
    int64_t move0;               // first of its entries in `moves`: at most min(budget, n_kv - budget) rows move
    int32_t n_kv, budget;
    int32_t index;               // its place in the caller's batch (kv_len)
};
struct EvictArgs {
    void *k, *v;
    int64_t row_bytes;
    const int32_t *pos, *kv_len;
    const float* mass;
    int32_t *pos_out, *kept_idx, *kv_len_out;
    float* mass_out;
    int32_t n_sink, n_recent, n_seq, max_moves;    // max_moves: the most rows that move in one sequence
    int2* moves;                 // workspace: (from, to) rows relative to kv_row
    int32_t* n_moves;            // workspace: [n_seq]
    EvictSeq s[kMaxBatch];
};
cudaError_t launch_cache_evict(const EvictArgs& a, cudaStream_t stream);

}  // namespace mvla
