// C-ABI layer of the calls on a cache in pages: argument validation, plans and workspaces, launch sequencing.  No stream
// synchronisation anywhere.
#include "page.h"
#include "page_checks.h"

#include <cstring>

using namespace mvla;

namespace {

PagePool pool_of(const CtxView& v, const mvla_pages& p, const int32_t* table, int64_t table_stride)
{
    PagePool q;
    q.k = p.k;
    q.v = p.v;
    q.k_scale = p.k_scale;
    q.v_scale = p.v_scale;
    q.table = table;
    q.table_stride = table_stride;
    q.n_pages = p.n_pages;
    q.page_shift = __builtin_ctz(static_cast<unsigned>(p.page_rows));
    q.kv_heads = v.kv_heads;
    q.head_dim = v.head_dim;
    return q;
}

// (head_dim, heads, rows) of the queries, in boxes of 64 elements of `pack` heads of 128 / pack rows: rows of 128 bytes in shared memory, 128-byte swizzle.
bool query_map(const CtxView& v, CUtensorMap* m, const void* q, int64_t rows, int pack)
{
    const cuuint64_t line = static_cast<cuuint64_t>(v.head_dim) * 2, dims[3] = {static_cast<cuuint64_t>(v.head_dim), static_cast<cuuint64_t>(v.n_heads), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[2] = {line, line * v.n_heads};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(pack), static_cast<cuuint32_t>(128 / pack)}, step[3] = {1, 1, 1};
    return v.encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// (head_dim, rows of a page, pages x key heads), in boxes of 64 elements of as many rows as a page has, 64 at most.  A pool without pages: a map that stands on
// `other` and is only asked for what lies outside of it.
bool page_map(const CtxView& v, CUtensorMap* m, const void* p, const void* other, int64_t pages, int page_rows)
{
    const cuuint64_t line = static_cast<cuuint64_t>(v.head_dim) * 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(v.head_dim), static_cast<cuuint64_t>(page_rows), static_cast<cuuint64_t>(pages > 0 ? pages * v.kv_heads : 1)};
    const cuuint64_t strides[2] = {line, line * page_rows};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(page_rows < kPageTile ? page_rows : kPageTile), 1}, step[3] = {1, 1, 1};
    return v.encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(pages > 0 ? p : other), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int32_t rows_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_page_rows* a, bool write, void* stream)
{
    if (!ctx || !a) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_page_rows(v, batch, seqs, a, write);
    if (rc != MVLA_OK) return rc;
    PageRowsArgs k;
    std::memset(&k, 0, sizeof k);
    int32_t total = 0;
    for (int b = 0; b < batch; ++b) {
        k.s[b] = PageSeq{seqs[b].q_row, seqs[b].n_q, seqs[b].n_kv, total, b};
        total += seqs[b].n_q;
    }
    if (total == 0 || (!a->k && !a->v)) return MVLA_OK;
    DeviceGuard guard(v.device);
    if (!guard.ok) return MVLA_ERR_CUDA;
    note_work(ctx);
    k.pool = pool_of(v, a->pages, a->table, a->table_stride);
    k.kv_len = a->kv_len;
    k.k = a->k;
    k.v = a->v;
    k.k_stride = a->k_stride;
    k.v_stride = a->v_stride;
    k.n_seq = batch;
    k.total = total;
    k.k_head = k.v_head = v.head_dim;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return close_call(ctx, write ? launch_page_write(v.hidden_dtype, a->pages.kind, k, st) : launch_page_read(v.hidden_dtype, a->pages.kind, k, st));
}

int32_t workspace_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* a, int64_t* bytes)
{
    if (!ctx || !a || !bytes) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_page_attention(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    *bytes = plan_page_attention(v, batch, seqs, a).bytes;
    return MVLA_OK;
}

int32_t attention_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* a, void* stream)
{
    if (!ctx || !a) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_page_attention(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    const PageAttendPlan plan = plan_page_attention(v, batch, seqs, a);
    if (plan.attend.total_q == 0) return MVLA_OK;
    rc = check_page_attention_memory(v, batch, a, plan);
    if (rc != MVLA_OK) return rc;
    DeviceGuard guard(v.device);
    if (!guard.ok) return MVLA_ERR_CUDA;
    note_work(ctx);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char* const ws = static_cast<char*>(a->workspace);
    mvla_attention w = as_window(a);
    w.workspace = a->workspace;
    w.workspace_bytes = plan.attend.bytes;
    CtxView h = v;
    static_cast<ServeShape&>(h) = hidden_shape(v);
    AttArgs t;
    fill_attention(t, h, batch, seqs, &w, plan.attend);
    const PagePool pool = pool_of(v, a->pages, a->table, a->table_stride);
    if (plan.attend.form == kFormToken) {
        cudaError_t e = launch_page_token(a->pages.kind, t, pool, plan.attend.rows, st);
        if (e == cudaSuccess && plan.attend.splits > 1) e = launch_attend_finish(t, st);
        return close_call(ctx, e);
    }
    t.k = a->pages.k;
    t.v = a->pages.v;
    t.table = a->table;
    t.table_stride = a->table_stride;
    t.n_pages = static_cast<int32_t>(a->pages.n_pages);
    t.page_shift = pool.page_shift;
    if (plan.dense_tiles > 0) {
        // the tiles that the queries see, one after another: pages of 64 rows, in order
        PageRowsArgs k;
        std::memset(&k, 0, sizeof k);
        int32_t tile = 0;
        for (int b = 0; b < batch; ++b) {
            k.s[b] = PageSeq{0, seqs[b].n_q, seqs[b].n_kv, tile * kPageTile, b};
            t.s[b].km_row = tile;
            tile += static_cast<int32_t>(seen_tiles(seqs[b], a->window, a->n_sink));
        }
        k.pool = pool;
        k.kv_len = a->kv_len;
        k.k = ws + plan.dense_k;
        k.v = ws + plan.dense_v;
        k.k_stride = k.v_stride = v.head_dim;
        k.k_head = k.v_head = static_cast<int64_t>(kPageTile) * v.head_dim;
        k.n_seq = batch;
        k.total = tile * kPageTile;
        k.window = t.window;
        k.n_sink = t.n_sink;
        const cudaError_t e = launch_page_tiles(v.hidden_dtype, a->pages.kind, k, st);
        if (e != cudaSuccess) return close_call(ctx, e);
        t.k = k.k;
        t.v = k.v;
        t.table = nullptr;
        t.n_pages = tile;
        t.page_shift = __builtin_ctz(kPageTile);
    }
    cudaError_t e;
    if (plan.unpack) {
        e = launch_page_decode(a->pages.kind, plan.unpack, t, pool, st);
    } else if (plan.attend.form == kFormFma) {
        e = launch_page_fma(t, st);
    } else {
        bool tokens = false;
        for (int b = 0; b < batch; ++b) {
            tokens |= seqs[b].n_q > 0 && static_cast<int64_t>(seqs[b].n_q) * (v.n_heads / v.kv_heads) <= kTokenRows;
            t.s[b].qm_row = static_cast<int32_t>(seqs[b].q_row);
        }
        AttMaps maps;
        if (!query_map(v, &maps.q, a->q, a->q_rows, plan.attend.pack) || !page_map(v, &maps.k, t.k, a->q, t.n_pages, 1 << t.page_shift) ||
            !page_map(v, &maps.v, t.v, a->q, t.n_pages, 1 << t.page_shift))
            return MVLA_ERR_CUDA;
        e = launch_page_tile(tokens, t, maps, st);
    }
    if (e == cudaSuccess && plan.attend.splits > 1) e = launch_attend_join(h.dtype, joined_by_ctas(h, plan.attend), t, st);
    return close_call(ctx, e);
}

long long ll(int64_t x) { return static_cast<long long>(x); }

}  // namespace

extern "C" {

int32_t mvla_page_write(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_page_rows* args, void* stream)
{
    ApiRange range("mvla_page_write");
    const int32_t rc = rows_impl(ctx, batch, seqs, args, true, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_page_write(batch %lld, kind %lld) -> %d\n", ll(batch), ll(args ? args->pages.kind : -1), rc);
    return rc;
}

int32_t mvla_page_read(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_page_rows* args, void* stream)
{
    ApiRange range("mvla_page_read");
    const int32_t rc = rows_impl(ctx, batch, seqs, args, false, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_page_read(batch %lld, kind %lld) -> %d\n", ll(batch), ll(args ? args->pages.kind : -1), rc);
    return rc;
}

int32_t mvla_page_attention(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* args, void* stream)
{
    ApiRange range("mvla_page_attention");
    const int32_t rc = attention_impl(ctx, batch, seqs, args, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_page_attention(batch %lld, kind %lld, window %lld) -> %d\n", ll(batch), ll(args ? args->pages.kind : -1), ll(args ? args->window : -1), rc);
    return rc;
}

int32_t mvla_page_attention_workspace(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* args, int64_t* bytes)
{
    ApiRange range("mvla_page_attention_workspace");
    const int32_t rc = workspace_impl(ctx, batch, seqs, args, bytes);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_page_attention_workspace(batch %lld) -> %d\n", ll(batch), rc);
    return rc;
}

}  // extern "C"
