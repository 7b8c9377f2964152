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
    k.packed_row = -1;
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
    if (plan.attend.form == kFormToken && plan.dense_k < 0) {
        AttArgs t;
        fill_attention(t, h, batch, seqs, &w, plan.attend);
        cudaError_t e = launch_page_token(a->pages.kind, t, pool_of(v, a->pages, a->table, a->table_stride), plan.attend.rows, st);
        if (e == cudaSuccess && plan.attend.splits > 1) e = launch_attend_finish(t, st);
        return close_call(ctx, e);
    }
    // the sequences' rows, packed one after another
    mvla_seq dense[kMaxBatch];
    PageRowsArgs k;
    std::memset(&k, 0, sizeof k);
    int32_t row = 0;
    for (int b = 0; b < batch; ++b) {
        dense[b] = seqs[b];
        dense[b].kv_row = row;
        k.s[b] = PageSeq{0, seqs[b].n_kv, seqs[b].n_kv, row, b};
        row += seqs[b].n_kv;
    }
    w.k = k.k = ws + plan.dense_k;
    w.v = k.v = ws + plan.dense_v;
    w.kv_rows = row;
    k.pool = pool_of(v, a->pages, a->table, a->table_stride);
    k.kv_len = a->kv_len;
    k.k_stride = k.v_stride = static_cast<int64_t>(v.kv_heads) * v.head_dim;
    k.n_seq = batch;
    k.total = row;
    k.from_start = 1;
    const cudaError_t e = row > 0 ? launch_page_read(v.hidden_dtype, a->pages.kind, k, st) : cudaSuccess;
    if (e != cudaSuccess) return close_call(ctx, e);
    return enqueue_attention(ctx, h, batch, dense, &w, plan.attend, st);
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
