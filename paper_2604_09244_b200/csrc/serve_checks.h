// Host-side checks and plans of the calls around the prune point: arithmetic on descriptors and addresses, without a device.
#pragma once

#include "attend_plan.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace mvla {

struct Range {
    const char* lo;
    const char* hi;
};
inline Range range_of(const void* p, int64_t bytes)
{
    const char* c = static_cast<const char*>(p);
    return {c, c ? c + bytes : c};
}
inline bool meet(const Range& a, const Range& b) { return a.lo && b.lo && a.lo < b.hi && b.lo < a.hi; }

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int32_t kMaxRows = 1 << 30;          // rows of one sequence, queries of one call
constexpr int64_t kMaxTensorRows = int64_t(1) << 36;   // rows of a tensor: products of sizes stay below 64 bits
constexpr int64_t kMaxStride = int64_t(1) << 30;

// Runs of rows [first, first + n) of a batch: whether two of them share a row.
template <class First, class Count>
bool shared_rows(int32_t batch, const mvla_seq* s, First first, Count count)
{
    bool ascending = true;
    int64_t end = 0;
    for (int b = 0; b < batch && ascending; ++b) {
        if (count(s[b]) == 0) continue;
        ascending = first(s[b]) >= end;
        end = first(s[b]) + count(s[b]);
    }
    if (ascending) return false;
    for (int b = 0; b < batch; ++b)
        for (int c = b + 1; c < batch; ++c)
            if (count(s[b]) && count(s[c]) && first(s[b]) < first(s[c]) + count(s[c]) && first(s[c]) < first(s[b]) + count(s[b])) return true;
    return false;
}

inline int32_t check_batch(const ServeShape& v, int32_t batch, const mvla_seq* seqs)
{
    if (batch < 1 || !seqs) return MVLA_ERR_INVALID_ARG;
    if (batch > v.max_batch) return MVLA_ERR_CAPACITY;
    for (int b = 0; b < batch; ++b) {
        const mvla_seq& s = seqs[b];
        if (s.n_kv < 0 || s.n_q < 0 || s.kv_row < 0 || s.q_row < 0 || s.budget < 0) return MVLA_ERR_INVALID_ARG;
        if (s.n_kv > kMaxRows || s.n_q > kMaxRows) return MVLA_ERR_UNSUPPORTED;
    }
    return MVLA_OK;
}

// ---- norms and rotation

// The norm's constant as the kernel takes it: where it is not zero, no smaller than the normal numbers of 32 bits (a row of zeros stays zeros), and infinite
// above them (all that is normed is nothing then).
inline float norm_eps(double eps)
{
    if (eps > FLT_MAX) return HUGE_VALF;
    return eps > 0.0 ? std::max(static_cast<float>(eps), FLT_MIN) : 0.f;
}

inline int32_t check_rope(const ServeShape& v, const mvla_qk_rope* r)
{
    if (r->n_rows < 0 || r->n_rows > 0x7FFFFFFF || r->kv_rows < 0 || r->kv_rows > kMaxTensorRows ||
        (r->flags & ~(MVLA_ROPE_NORM | MVLA_ROPE_INTERLEAVED)))
        return MVLA_ERR_INVALID_ARG;
    if (r->rot_dim < 0 || r->rot_dim > v.head_dim || !(r->eps >= 0.0) || !std::isfinite(r->eps)) return MVLA_ERR_INVALID_ARG;
    if (r->rot_dim % 16 != 0) return MVLA_ERR_UNSUPPORTED;
    if (r->n_rows == 0) return MVLA_OK;                    // (tensors without rows may have no address where their outputs, a cache, have one)
    if (r->rot_dim > 0 && (!r->pos || !r->inv_freq)) return MVLA_ERR_INVALID_ARG;
    if (!aligned(r->pos, 4) || !aligned(r->out_rows, 4) || !aligned(r->inv_freq, 8)) return MVLA_ERR_INVALID_ARG;
    if (!(r->flags & MVLA_ROPE_NORM) && (r->q_weight || r->k_weight)) return MVLA_ERR_INVALID_ARG;
    if (!aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return MVLA_ERR_INVALID_ARG;
    if ((r->k || r->v) && !r->out_rows && r->kv_rows < r->n_rows) return MVLA_ERR_INVALID_ARG;
    const void* in[3] = {r->q, r->k, r->v};
    void* out[3] = {r->q_out, r->k_out, r->v_out};
    const int64_t stride[3] = {r->q_stride, r->k_stride, r->v_stride};
    const int64_t wide = static_cast<int64_t>(v.wide), elem = static_cast<int64_t>(v.elem);
    // everything a call reads besides: the weights, positions, frequencies, destinations
    const Range side[5] = {range_of(r->q_weight, v.head_dim * wide), range_of(r->k_weight, v.head_dim * wide),
                           range_of(r->rot_dim ? r->pos : nullptr, r->n_rows * 4), range_of(r->rot_dim ? r->inv_freq : nullptr, r->rot_dim * 4),
                           range_of(r->out_rows, r->n_rows * 4)};
    Range ri[3], ro[3];
    for (int i = 0; i < 3; ++i) {
        const int64_t width = static_cast<int64_t>(i ? v.kv_heads : v.n_heads) * v.head_dim;
        if ((in[i] == nullptr) != (out[i] == nullptr)) return MVLA_ERR_INVALID_ARG;
        ri[i] = ro[i] = Range{nullptr, nullptr};
        if (!in[i]) continue;
        if (!aligned(in[i], 16) || !aligned(out[i], 16) || stride[i] < 0 || stride[i] > kMaxStride || (r->n_rows > 1 && stride[i] < width) ||
            stride[i] * wide % 16 != 0)
            return MVLA_ERR_INVALID_ARG;
        ri[i] = range_of(in[i], ((r->n_rows - 1) * stride[i] + width) * wide);
        ro[i] = range_of(out[i], (i ? r->kv_rows : r->n_rows) * width * elem);
    }
    for (int i = 0; i < 3; ++i) {
        const int64_t width = static_cast<int64_t>(i ? v.kv_heads : v.n_heads) * v.head_dim;
        for (int j = 0; j < 3; ++j) {
            const bool itself = i == j && in[i] == out[i] && v.elem == v.wide && (i == 0 || !r->out_rows) && (r->n_rows <= 1 || stride[i] == width);
            if (meet(ro[i], ri[j]) && !itself) return MVLA_ERR_INVALID_ARG;
            if (i < j && meet(ro[i], ro[j])) return MVLA_ERR_INVALID_ARG;
        }
        for (const Range& s : side) if (meet(ro[i], s)) return MVLA_ERR_INVALID_ARG;
    }
    return MVLA_OK;
}

// ---- windowed attention

// The scale of the dot products in powers of two, as the kernels take it.
inline double scale_log2(const ServeShape& v, const mvla_attention* a)
{
    return (a->scale > 0.0 ? a->scale : 1.0 / std::sqrt(static_cast<double>(v.head_dim))) * 1.4426950408889634;       // log2 e
}

inline int32_t check_attention(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_attention* a)
{
    const int32_t rc = check_batch(v, batch, seqs);
    if (rc != MVLA_OK) return rc;
    if (a->window < 1 || a->n_sink < 0 || !(a->scale >= 0.0)) return MVLA_ERR_INVALID_ARG;
    // (a normal number of 32 bits: zero times the -infinity of a row that is not seen is no number)
    if (!(scale_log2(v, a) >= FLT_MIN && scale_log2(v, a) <= FLT_MAX)) return MVLA_ERR_INVALID_ARG;
    if (a->kv_pos && !a->q_pos) return MVLA_ERR_INVALID_ARG;
    if (a->q_rows < 0 || a->kv_rows < 0 || a->q_rows > kMaxTensorRows || a->kv_rows > kMaxTensorRows) return MVLA_ERR_INVALID_ARG;
    if (v.kv_heads > 65535) return MVLA_ERR_UNSUPPORTED;
    int64_t total_q = 0, total_kv = 0;
    for (int b = 0; b < batch; ++b) {
        const mvla_seq& s = seqs[b];
        if (s.q_row > a->q_rows - s.n_q || s.kv_row > a->kv_rows - s.n_kv) return MVLA_ERR_INVALID_ARG;
        total_q += s.n_q;
        total_kv += s.n_kv;
    }
    if (v.dtype != MVLA_DTYPE_FP32 && (a->q_rows > 0x7FFFFFFF || a->kv_rows > 0x7FFFFFFF)) return MVLA_ERR_UNSUPPORTED;   // (rows of a tensor map are counted in 32 bits)
    if (total_q * v.n_heads / v.kv_heads > kMaxRows || total_kv > 0x7FFFFFFF) return MVLA_ERR_UNSUPPORTED;
    if (shared_rows(batch, seqs, [](const mvla_seq& s) { return s.q_row; }, [](const mvla_seq& s) { return s.n_q; })) return MVLA_ERR_INVALID_ARG;
    if (a->mass && shared_rows(batch, seqs, [](const mvla_seq& s) { return s.kv_row; }, [](const mvla_seq& s) { return s.n_kv; }))
        return MVLA_ERR_INVALID_ARG;
    return MVLA_OK;
}

// Whether every position is known to the host.
inline bool all_counted(const mvla_attention* a) { return !a->q_pos && !a->kv_pos && !a->kv_len; }
inline AttendPlan plan_of(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_attention* a)
{
    return plan_attend(v, batch, seqs, all_counted(a), a->window, a->n_sink, a->mass != nullptr);
}

// Pointers of a call that has queries.
inline int32_t check_attention_memory(const ServeShape& v, int32_t batch, const mvla_attention* a, const AttendPlan& plan)
{
    if (!a->q || !a->out || (plan.total_kv > 0 && (!a->k || !a->v))) return MVLA_ERR_INVALID_ARG;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->out, 16) || !aligned(a->lse, 4) || !aligned(a->mass, 4) ||
        !aligned(a->q_pos, 4) || !aligned(a->kv_pos, 4) || !aligned(a->kv_len, 4) || !aligned(a->workspace, 256))
        return MVLA_ERR_INVALID_ARG;
    if (plan.bytes > 0 && (!a->workspace || a->workspace_bytes < plan.bytes)) return MVLA_ERR_INVALID_ARG;
    const int64_t qw = static_cast<int64_t>(v.n_heads) * v.head_dim, kw = static_cast<int64_t>(v.kv_heads) * v.head_dim;
    const int64_t elem = static_cast<int64_t>(v.elem), wide = static_cast<int64_t>(v.wide);
    const Range in[6] = {range_of(a->q, a->q_rows * qw * elem), range_of(a->k, a->kv_rows * kw * elem), range_of(a->v, a->kv_rows * kw * elem),
                         range_of(a->q_pos, a->q_rows * 4), range_of(a->kv_pos, a->kv_rows * 4), range_of(a->kv_len, batch * 4)};
    const Range out[4] = {range_of(a->out, a->q_rows * qw * wide), range_of(a->lse, a->q_rows * v.n_heads * 4), range_of(a->mass, a->kv_rows * 4),
                          range_of(plan.bytes ? a->workspace : nullptr, plan.bytes)};
    for (int i = 0; i < 4; ++i) {
        for (const Range& r : in) if (meet(out[i], r)) return MVLA_ERR_INVALID_ARG;
        for (int j = i + 1; j < 4; ++j) if (meet(out[i], out[j])) return MVLA_ERR_INVALID_ARG;
    }
    return MVLA_OK;
}

// ---- eviction

struct EvictPlan {
    int64_t moves = 0;           // rows that may move in all
    int32_t most = 0;            // ... in one sequence
    int64_t count_at = 0, bytes = 0;
};
inline int64_t moves_of(const mvla_seq& s) { return std::min<int64_t>(s.budget, std::max(0, s.n_kv - s.budget)); }
inline EvictPlan plan_evict(int32_t batch, const mvla_seq* seqs)
{
    EvictPlan p;
    for (int b = 0; b < batch; ++b) {
        const int64_t n = moves_of(seqs[b]);
        p.moves += n;
        p.most = std::max(p.most, static_cast<int32_t>(n));
    }
    Workspace w;
    w.take(p.moves * 2 * static_cast<int64_t>(sizeof(int32_t)));
    p.count_at = w.take(batch * static_cast<int64_t>(sizeof(int32_t)));
    p.bytes = w.bytes;
    return p;
}

inline int32_t check_eviction(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_eviction* a)
{
    const int32_t rc = check_batch(v, batch, seqs);
    if (rc != MVLA_OK) return rc;
    if (a->n_sink < 0 || a->n_recent < 0 || a->kv_rows < 0 || a->kv_rows > kMaxTensorRows) return MVLA_ERR_INVALID_ARG;
    for (int b = 0; b < batch; ++b)
        if (seqs[b].kv_row > a->kv_rows - seqs[b].n_kv || static_cast<int64_t>(a->n_sink) + a->n_recent > seqs[b].budget) return MVLA_ERR_INVALID_ARG;
    if (shared_rows(batch, seqs, [](const mvla_seq& s) { return s.kv_row; }, [](const mvla_seq& s) { return s.n_kv; })) return MVLA_ERR_INVALID_ARG;
    return MVLA_OK;
}

inline int32_t check_eviction_memory(const ServeShape& v, int32_t batch, const mvla_eviction* a, const EvictPlan& plan)
{
    // (a cache without rows may have no address: then only its lengths, which are zero, are written)
    if (a->kv_rows > 0 && (!a->k || !a->v || !a->pos || !a->mass || !a->pos_out || !a->mass_out)) return MVLA_ERR_INVALID_ARG;
    if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->pos, 4) || !aligned(a->mass, 4) || !aligned(a->pos_out, 4) || !aligned(a->mass_out, 4) ||
        !aligned(a->kept_idx, 4) || !aligned(a->kv_len, 4) || !aligned(a->kv_len_out, 4) || !aligned(a->workspace, 256))
        return MVLA_ERR_INVALID_ARG;
    if (!a->workspace || a->workspace_bytes < plan.bytes) return MVLA_ERR_INVALID_ARG;
    const int64_t row_bytes = static_cast<int64_t>(v.kv_heads) * v.head_dim * static_cast<int64_t>(v.elem), words = a->kv_rows * 4;
    const Range in[3] = {range_of(a->pos, words), range_of(a->mass, words), range_of(a->kv_len, batch * 4)};
    const Range out[7] = {range_of(a->pos_out, words), range_of(a->mass_out, words), range_of(a->kv_len_out, batch * 4), range_of(a->kept_idx, words),
                          range_of(a->k, a->kv_rows * row_bytes), range_of(a->v, a->kv_rows * row_bytes), range_of(a->workspace, plan.bytes)};
    for (int i = 0; i < 7; ++i) {
        for (int j = 0; j < 3; ++j) if (!(i == j && out[i].lo == in[j].lo) && meet(out[i], in[j])) return MVLA_ERR_INVALID_ARG;
        for (int j = i + 1; j < 7; ++j) if (meet(out[i], out[j])) return MVLA_ERR_INVALID_ARG;
    }
    return MVLA_OK;
}

}  // namespace mvla
