// C-ABI layer of the calls around the prune point: argument validation, plans and workspaces, launch sequencing.  No stream
// synchronisation anywhere.
#include "serve.h"
#include "serve_checks.h"

#include <cstring>

using namespace mvla;

namespace {

int32_t rope_impl(mvla_ctx* ctx, const mvla_qk_rope* r, void* stream)
{
    if (!ctx || !r) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_rope(v, r);
    if (rc != MVLA_OK) return rc;
    if (r->n_rows == 0 || (!r->q && !r->k && !r->v)) return MVLA_OK;
    DeviceGuard guard(v.device);
    if (!guard.ok) return MVLA_ERR_CUDA;
    note_work(ctx);
    RopeJob job;
    std::memset(&job, 0, sizeof job);
    job.q = r->q; job.k = r->k; job.v = r->v; job.q_weight = r->q_weight; job.k_weight = r->k_weight;
    job.n_rows = r->n_rows; job.q_stride = r->q_stride; job.k_stride = r->k_stride; job.v_stride = r->v_stride; job.kv_rows = r->kv_rows;
    job.pos = r->pos; job.inv_freq = r->inv_freq; job.out_rows = r->out_rows;
    job.q_out = r->q_out; job.k_out = r->k_out; job.v_out = r->v_out;
    job.n_heads = v.n_heads; job.kv_heads = v.kv_heads; job.head_dim = v.head_dim; job.rot_dim = r->rot_dim;
    job.eps = norm_eps(r->eps);
    job.norm = (r->flags & MVLA_ROPE_NORM) != 0;
    job.interleaved = (r->flags & MVLA_ROPE_INTERLEAVED) != 0;
    return close_call(ctx, launch_qk_norm_rope(v.dtype, job, static_cast<cudaStream_t>(stream)));
}

int32_t workspace_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_attention* a, int64_t* bytes)
{
    if (!ctx || !a || !bytes) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_attention(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    *bytes = plan_of(v, batch, seqs, a).bytes;
    return MVLA_OK;
}

// (head_dim, heads, rows) of a token-major tensor, in boxes of 64 elements x `box_heads` x `box_rows`: rows of 128 bytes in shared memory,
// 128-byte swizzle, heads of a token next to one another.
bool row_map(const CtxView& v, CUtensorMap* m, const void* p, int heads, int64_t rows, int box_heads, int box_rows)
{
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(v.head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(v.head_dim) * 2, static_cast<cuuint64_t>(v.head_dim) * 2 * heads};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_rows)}, step[3] = {1, 1, 1};
    return v.encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The tile form: tensor maps over the caller's bf16 rows, or over their widened copies.
int32_t attend_by_tiles(const CtxView& v, AttArgs& k, const mvla_attention* a, const AttendPlan& plan, cudaError_t* e, cudaStream_t st)
{
    const bool widen = plan.wide_q >= 0;
    char* const ws = static_cast<char*>(a->workspace);
    const void* const q = widen ? ws + plan.wide_q : a->q;
    const void* const kk = widen ? ws + plan.wide_k : a->k;
    const void* const vv = widen ? ws + plan.wide_v : a->v;
    const int64_t q_rows = widen ? plan.total_q : a->q_rows, kv_rows = widen ? plan.total_kv : a->kv_rows;
    bool tokens = false;
    for (int b = 0; b < k.n_seq; ++b) {
        AttSeq& s = k.s[b];
        tokens |= !widen && s.n_q > 0 && static_cast<int64_t>(s.n_q) * (v.n_heads / v.kv_heads) <= kTokenRows;
        s.qm_row = widen ? s.qp0 : static_cast<int32_t>(s.q_row);
        s.km_row = widen ? s.kvp0 : static_cast<int32_t>(s.kv_row);
    }
    AttMaps maps;
    std::memset(&maps, 0, sizeof maps);
    constexpr int kKeys = 64;              // of a tile (attend_tile.cu)
    if (!row_map(v, &maps.q, q, v.n_heads, q_rows, plan.pack, 128 / plan.pack)) return MVLA_ERR_CUDA;
    // (no cached rows: no key tile is ever asked for)
    if (plan.total_kv > 0 && (!row_map(v, &maps.k, kk, v.kv_heads, kv_rows, 1, kKeys) || !row_map(v, &maps.v, vv, v.kv_heads, kv_rows, 1, kKeys))) return MVLA_ERR_CUDA;
    *e = widen ? launch_widen(k, ws + plan.wide_q, ws + plan.wide_k, ws + plan.wide_v, st) : cudaSuccess;
    if (*e == cudaSuccess) *e = launch_attend_tile(widen, tokens, k, maps, st);
    if (*e == cudaSuccess && plan.splits > 1) *e = launch_attend_join(v.dtype, plan.splits > kFewParts, k, st);
    if (*e == cudaSuccess && a->mass && plan.total_kv > 0) {
        if (!row_map(v, &maps.k, kk, v.kv_heads, kv_rows, 1, 128)) return MVLA_ERR_CUDA;
        *e = launch_attend_weights(widen, k, maps, st);
    }
    return MVLA_OK;
}

}  // namespace

namespace mvla {

void fill_attention(AttArgs& k, const CtxView& v, int32_t batch, const mvla_seq* seqs, const mvla_attention* a, const AttendPlan& plan)
{
    std::memset(&k, 0, sizeof k);
    k.q = a->q; k.k = a->k; k.v = a->v; k.out = a->out; k.lse = a->lse; k.mass = a->mass;
    k.q_pos = a->q_pos; k.kv_pos = a->kv_pos; k.kv_len = a->kv_len;
    k.n_heads = v.n_heads; k.kv_heads = v.kv_heads; k.head_dim = v.head_dim; k.window = a->window;
    // (no window: the one distance that is not below MVLA_WINDOW_ALL, from the last position that there is to the first, is a sink's)
    k.n_sink = a->window == MVLA_WINDOW_ALL && a->n_sink == 0 ? 1 : a->n_sink;
    k.scale_log2 = static_cast<float>(scale_log2(v, a));
    k.n_seq = batch; k.n_blocks = static_cast<int32_t>(plan.blocks);
    k.total_q = static_cast<int32_t>(plan.total_q); k.total_kv = static_cast<int32_t>(plan.total_kv);
    k.splits = plan.splits; k.mass_parts = plan.mass_parts; k.pack = plan.pack; k.status = v.status_dev;
    char* const ws = static_cast<char*>(a->workspace);
    const auto at = [&](int64_t off) { return off < 0 ? nullptr : ws + off; };
    k.part_o = reinterpret_cast<float*>(at(plan.part_o));
    k.part_ml = reinterpret_cast<float2*>(at(plan.part_ml));
    k.lse2 = reinterpret_cast<float*>(at(plan.lse2));
    k.part_mass = reinterpret_cast<float*>(at(plan.part_mass));
    k.logits = reinterpret_cast<float*>(at(plan.logits));
    k.cluster = plan.cluster;
    k.skip_whole = plan.form == kFormToken || plan.form == kFormPageTile;
    const int group = v.n_heads / v.kv_heads;
    const bool counted = all_counted(a);
    int32_t blk = 0, qp = 0, kvp = 0, tile = 0;
    int64_t part = 0, logit = 0;
    for (int b = 0; b < batch; ++b) {
        const mvla_seq& s = seqs[b];
        const int32_t parts = parts_of(plan, s, counted, a->window, a->n_sink);
        k.s[b] = AttSeq{s.q_row, s.kv_row, s.n_q, s.n_kv, blk, qp, kvp, tile, parts, part, logit, 0, 0, b};
        blk += plan.form == kFormToken ? parts * plan.cluster
             : plan.form == kFormPageTile ? static_cast<int32_t>((static_cast<int64_t>(s.n_q) + plan.queries - 1) / plan.queries * parts)
             : static_cast<int32_t>(plan.form == kFormTile ? (static_cast<int64_t>(s.n_q) + plan.queries - 1) / plan.queries
                                                           : (static_cast<int64_t>(s.n_q) * group + plan.rows - 1) / plan.rows);
        qp += s.n_q;
        kvp += s.n_kv;
        tile += static_cast<int32_t>((static_cast<int64_t>(s.n_kv) + 127) / 128);
        part += static_cast<int64_t>(parts) * s.n_q;
        logit += static_cast<int64_t>(s.n_q) * v.n_heads * s.n_kv;
    }
}

}  // namespace mvla

namespace {

int32_t attention_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_attention* a, void* stream)
{
    if (!ctx || !a) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_attention(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    const AttendPlan plan = plan_of(v, batch, seqs, a);
    if (plan.total_q == 0) return MVLA_OK;
    rc = check_attention_memory(v, batch, a, plan);
    if (rc != MVLA_OK) return rc;
    DeviceGuard guard(v.device);
    if (!guard.ok) return MVLA_ERR_CUDA;
    note_work(ctx);
    AttArgs k;
    fill_attention(k, v, batch, seqs, a, plan);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (plan.form == kFormTile) {
        rc = attend_by_tiles(v, k, a, plan, &e, st);
        if (rc != MVLA_OK) return rc;
    } else if (plan.form == kFormToken) {
        e = launch_attend_token(v.dtype, k, plan.rows, st);
        if (e == cudaSuccess && (plan.splits > 1 || a->mass)) e = launch_attend_finish(k, st);
        return close_call(ctx, e);
    } else {
        e = launch_attend_fma(k, plan.rows, st);
        if (e == cudaSuccess && plan.splits > 1) e = launch_attend_join(v.dtype, plan.splits > kFewParts, k, st);
        if (e == cudaSuccess && a->mass) e = launch_mass_fma(k, st);
    }
    if (e == cudaSuccess && a->mass) e = launch_mass_add(k, st);
    return close_call(ctx, e);
}

int32_t evict_workspace_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_eviction* a, int64_t* bytes)
{
    if (!ctx || !a || !bytes) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_eviction(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    *bytes = plan_evict(batch, seqs).bytes;
    return MVLA_OK;
}

int32_t evict_impl(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_eviction* a, void* stream)
{
    if (!ctx || !a) return MVLA_ERR_INVALID_ARG;
    CtxView v;
    int32_t rc = open_call(ctx, &v);
    if (rc == MVLA_OK) rc = check_eviction(v, batch, seqs, a);
    if (rc != MVLA_OK) return rc;
    const EvictPlan plan = plan_evict(batch, seqs);
    rc = check_eviction_memory(v, batch, a, plan);
    if (rc != MVLA_OK) return rc;
    DeviceGuard guard(v.device);
    if (!guard.ok) return MVLA_ERR_CUDA;
    note_work(ctx);
    EvictArgs k;
    std::memset(&k, 0, sizeof k);
    k.k = a->k; k.v = a->v;
    k.row_bytes = static_cast<int64_t>(v.kv_heads) * v.head_dim * static_cast<int64_t>(v.elem);
    k.pos = a->pos; k.kv_len = a->kv_len; k.mass = a->mass;
    k.pos_out = a->pos_out; k.kept_idx = a->kept_idx; k.kv_len_out = a->kv_len_out; k.mass_out = a->mass_out;
    k.n_sink = a->n_sink; k.n_recent = a->n_recent; k.n_seq = batch; k.max_moves = plan.most;
    k.moves = static_cast<int2*>(a->workspace);
    k.n_moves = reinterpret_cast<int32_t*>(static_cast<char*>(a->workspace) + plan.count_at);
    int64_t at = 0;
    for (int b = 0; b < batch; ++b) {
        k.s[b] = EvictSeq{seqs[b].kv_row, at, seqs[b].n_kv, seqs[b].budget, b};
        at += moves_of(seqs[b]);
    }
    return close_call(ctx, launch_cache_evict(k, static_cast<cudaStream_t>(stream)));
}

long long ll(int64_t x) { return static_cast<long long>(x); }

}  // namespace

extern "C" {

int32_t mvla_qk_norm_rope(mvla_ctx* ctx, const mvla_qk_rope* args, void* stream)
{
    ApiRange range("mvla_qk_norm_rope");
    const int32_t rc = rope_impl(ctx, args, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_qk_norm_rope(rows %lld, rot_dim %lld, flags %lld) -> %d\n", ll(args ? args->n_rows : -1), ll(args ? args->rot_dim : -1), ll(args ? args->flags : 0), rc);
    return rc;
}

int32_t mvla_window_attention(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_attention* args, void* stream)
{
    ApiRange range("mvla_window_attention");
    const int32_t rc = attention_impl(ctx, batch, seqs, args, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_window_attention(batch %lld, window %lld, sinks %lld) -> %d\n", ll(batch), ll(args ? args->window : -1), ll(args ? args->n_sink : -1), rc);
    return rc;
}

int32_t mvla_window_attention_workspace(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_attention* args, int64_t* bytes)
{
    ApiRange range("mvla_window_attention_workspace");
    const int32_t rc = workspace_impl(ctx, batch, seqs, args, bytes);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_window_attention_workspace(batch %lld) -> %d\n", ll(batch), rc);
    return rc;
}

int32_t mvla_cache_evict(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_eviction* args, void* stream)
{
    ApiRange range("mvla_cache_evict");
    const int32_t rc = evict_impl(ctx, batch, seqs, args, stream);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_cache_evict(batch %lld, sinks %lld, recent %lld) -> %d\n", ll(batch), ll(args ? args->n_sink : -1), ll(args ? args->n_recent : -1), rc);
    return rc;
}

int32_t mvla_cache_evict_workspace(mvla_ctx* ctx, int32_t batch, const mvla_seq* seqs, const mvla_eviction* args, int64_t* bytes)
{
    ApiRange range("mvla_cache_evict_workspace");
    const int32_t rc = evict_workspace_impl(ctx, batch, seqs, args, bytes);
    if (log_enabled()) std::fprintf(stderr, "[mvla] mvla_cache_evict_workspace(batch %lld) -> %d\n", ll(batch), rc);
    return rc;
}

}  // extern "C"
