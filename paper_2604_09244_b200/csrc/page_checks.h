// Host-side checks and plans of the calls on a cache in pages: arithmetic on descriptors and addresses, without a device.
#pragma once

#include "page_plan.h"
#include "serve_checks.h"

namespace mvla {

inline int64_t page_data_bytes(const ServeShape& v, const mvla_pages& p)
{
    return p.n_pages * v.kv_heads * p.page_rows * page_row_bytes(p.kind, v.head_dim, static_cast<int>(v.wide));
}
inline int64_t page_scale_bytes(const ServeShape& v, const mvla_pages& p)
{
    return p.n_pages * v.kv_heads * p.page_rows * page_row_scales(p.kind, v.head_dim);
}

// The sequences of a call, and the table that has to name their pages.
inline int32_t check_page_batch(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_pages& p, int64_t table_stride)
{
    const int32_t rc = check_batch(v, batch, seqs);
    if (rc != MVLA_OK) return rc;
    if (p.kind < MVLA_PAGE_ROWS || p.kind > MVLA_PAGE_E2M1 || p.n_pages < 0 || table_stride < 0 || table_stride > kMaxTensorRows) return MVLA_ERR_INVALID_ARG;
    if (p.page_rows < 16 || p.page_rows > 256 || (p.page_rows & (p.page_rows - 1))) return MVLA_ERR_UNSUPPORTED;
    if (p.n_pages > 0x7FFFFFFF || p.n_pages * v.kv_heads > 0x7FFFFFFF || v.kv_heads > 65535) return MVLA_ERR_UNSUPPORTED;
    int64_t rows = 0, cached = 0;
    for (int b = 0; b < batch; ++b) {
        const mvla_seq& s = seqs[b];
        if ((static_cast<int64_t>(s.n_kv) + p.page_rows - 1) / p.page_rows > table_stride) return MVLA_ERR_INVALID_ARG;
        rows += s.n_q;
        cached += s.n_kv;
    }
    if (rows > kMaxRows || cached > 0x7FFFFFFF) return MVLA_ERR_UNSUPPORTED;
    return MVLA_OK;
}

// The pool's own memory: there, aligned, its parts apart.  `parts` receives their ranges.
inline int32_t check_pool(const ServeShape& v, const mvla_pages& p, Range (&parts)[4])
{
    const bool scaled = p.kind != MVLA_PAGE_ROWS;
    if ((p.n_pages > 0 && (!p.k || !p.v || (scaled && (!p.k_scale || !p.v_scale)))) || (!scaled && (p.k_scale || p.v_scale))) return MVLA_ERR_INVALID_ARG;
    if (!aligned(p.k, 16) || !aligned(p.v, 16) || !aligned(p.k_scale, 16) || !aligned(p.v_scale, 16)) return MVLA_ERR_INVALID_ARG;
    const int64_t data = page_data_bytes(v, p), scale = page_scale_bytes(v, p);
    parts[0] = range_of(p.k, data);
    parts[1] = range_of(p.v, data);
    parts[2] = range_of(p.k_scale, scale);
    parts[3] = range_of(p.v_scale, scale);
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j) if (meet(parts[i], parts[j])) return MVLA_ERR_INVALID_ARG;
    return MVLA_OK;
}
inline Range table_range(int32_t batch, const int32_t* table, int64_t stride) { return range_of(stride > 0 ? table : nullptr, batch * stride * 4); }

// mvla_page_write (`write`) and mvla_page_read.
inline int32_t check_page_rows(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_page_rows* a, bool write)
{
    int32_t rc = check_page_batch(v, batch, seqs, a->pages, a->table_stride);
    if (rc != MVLA_OK) return rc;
    if (a->rows < 0 || a->rows > kMaxTensorRows) return MVLA_ERR_INVALID_ARG;
    int64_t total = 0, cached = 0;
    for (int b = 0; b < batch; ++b) {
        if (seqs[b].q_row > a->rows - seqs[b].n_q) return MVLA_ERR_INVALID_ARG;
        total += seqs[b].n_q;
        cached += seqs[b].n_kv;
    }
    if (!write && shared_rows(batch, seqs, [](const mvla_seq& s) { return s.q_row; }, [](const mvla_seq& s) { return s.n_q; })) return MVLA_ERR_INVALID_ARG;
    if (total == 0) return MVLA_OK;                        // (nothing to do: whatever the pointers are)
    Range pool[4];
    rc = check_pool(v, a->pages, pool);
    if (rc != MVLA_OK) return rc;
    if ((cached > 0 && !a->table) || !aligned(a->table, 4) || !aligned(a->kv_len, 4)) return MVLA_ERR_INVALID_ARG;
    const int64_t width = static_cast<int64_t>(v.kv_heads) * v.head_dim, wide = static_cast<int64_t>(v.wide);
    const void* const p[2] = {a->k, a->v};
    const int64_t stride[2] = {a->k_stride, a->v_stride};
    Range rows[2];
    for (int i = 0; i < 2; ++i) {
        rows[i] = Range{nullptr, nullptr};
        if (!p[i]) continue;
        if (!aligned(p[i], 16) || stride[i] < 0 || stride[i] > kMaxStride || (a->rows > 1 && stride[i] < width) || stride[i] * wide % 16 != 0) return MVLA_ERR_INVALID_ARG;
        rows[i] = range_of(p[i], ((a->rows - 1) * stride[i] + width) * wide);
    }
    // slices of a fused tensor interleave: of two outputs that do, rows must have room for one another
    const Range side[2] = {table_range(batch, a->table, a->table_stride), range_of(a->kv_len, batch * 4)};
    for (const Range& r : rows) {
        for (const Range& q : pool) if (meet(r, q)) return MVLA_ERR_INVALID_ARG;
        if (!write) for (const Range& q : side) if (meet(r, q)) return MVLA_ERR_INVALID_ARG;
    }
    if (write) {
        for (const Range& r : pool) for (const Range& q : side) if (meet(r, q)) return MVLA_ERR_INVALID_ARG;
    } else if (meet(rows[0], rows[1])) {
        const char* lo = rows[0].lo < rows[1].lo ? rows[0].lo : rows[1].lo;
        const int64_t apart = (rows[0].lo < rows[1].lo ? rows[1].lo : rows[0].lo) - lo;
        if (stride[0] != stride[1] || apart < width * wide || apart + width * wide > stride[0] * wide) return MVLA_ERR_INVALID_ARG;
    }
    return MVLA_OK;
}

// ---- attention over pages

constexpr int kPageTile = 64;                // keys of a tile (attend_tile.cu), rows of an unpacked one

// Whether CTAs join the parts of every (query, head): many parts, and no more CTAs than run at once.  us: 200 queries of 16 heads, 9 parts, 24 by CTAs, 7 by warps; 30 of 8
// heads of 128, 18 parts, 2 less by CTAs.
inline bool joined_by_ctas(const ServeShape& c, const AttendPlan& p) { return p.splits > kFewParts && p.total_q * c.n_heads <= 8 * static_cast<int64_t>(c.sm_count); }

struct PageAttendPlan {
    AttendPlan attend;
    // quantised pages that are no single tokens': the tiles that some query sees, as elements of the hidden type (-1: there are none)
    int64_t dense_k = -1, dense_v = -1, dense_tiles = 0, bytes = 0;
    int32_t unpack = 0;          // ... or the tile form unpacks them on the way, for so many tiles of query rows at a time
};

// Tiles that a sequence's queries see, at most.
inline int64_t seen_tiles(const mvla_seq& s, int32_t window, int32_t n_sink)
{
    if (s.n_q == 0) return 0;
    const int64_t all = (static_cast<int64_t>(s.n_kv) + kPageTile - 1) / kPageTile;
    const int64_t near = (static_cast<int64_t>(window) + s.n_q - 1 + kPageTile - 1) / kPageTile + 1, sinks = (static_cast<int64_t>(n_sink) + kPageTile - 1) / kPageTile;
    return std::min(all, near + sinks);
}

inline ServeShape hidden_shape(const ServeShape& v)
{
    ServeShape h = v;
    h.dtype = v.hidden_dtype;
    h.elem = v.wide;
    return h;
}

// The call as mvla_window_attention would be given it.
inline mvla_attention as_window(const mvla_paged_attention* a)
{
    mvla_attention w = {};
    w.q = a->q;
    w.q_rows = a->q_rows;
    w.kv_len = a->kv_len;
    w.window = a->window;
    w.n_sink = a->n_sink;
    w.scale = a->scale;
    w.out = a->out;
    w.lse = a->lse;
    return w;
}

inline int32_t check_page_attention(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* a)
{
    int32_t rc = check_page_batch(v, batch, seqs, a->pages, a->table_stride);
    if (rc != MVLA_OK) return rc;
    const ServeShape h = hidden_shape(v);
    const mvla_attention w = as_window(a);
    if (w.window < 1 || w.n_sink < 0 || !(w.scale >= 0.0)) return MVLA_ERR_INVALID_ARG;
    if (!(scale_log2(h, &w) >= FLT_MIN && scale_log2(h, &w) <= FLT_MAX)) return MVLA_ERR_INVALID_ARG;
    if (a->q_rows < 0 || a->q_rows > kMaxTensorRows) return MVLA_ERR_INVALID_ARG;
    int64_t total_q = 0;
    for (int b = 0; b < batch; ++b) {
        if (seqs[b].q_row > a->q_rows - seqs[b].n_q) return MVLA_ERR_INVALID_ARG;
        total_q += seqs[b].n_q;
    }
    if (h.dtype != MVLA_DTYPE_FP32 && a->q_rows > 0x7FFFFFFF) return MVLA_ERR_UNSUPPORTED;      // (rows of a tensor map are counted in 32 bits)
    if (total_q * v.n_heads / v.kv_heads > kMaxRows) return MVLA_ERR_UNSUPPORTED;
    if (shared_rows(batch, seqs, [](const mvla_seq& s) { return s.q_row; }, [](const mvla_seq& s) { return s.n_q; })) return MVLA_ERR_INVALID_ARG;
    return MVLA_OK;
}

// Parts (clusters of 1, 2, 4 or 8 CTAs) of about the same length over the whole batch, a multiple of 64 keys to a CTA, so that their CTAs fill whole rounds
// of those that fit, or a cluster to a sequence: what ends first, in keys of a CTA (about 30 a microsecond): its keys and 256 for its start and end in every round, 56 where a cluster joins
// (16 requests of one token over 30 to 100 rows 7.3 us in clusters, 5.3 without), and where a sequence has several clusters 128 for the kernel that joins them and 4 for every one of the most there are (one token over 131072 e4m3 rows: the join 7.3 us
// of 68 with 74 parts).  256 parts to a sequence at most.
inline void cut_page_tokens(AttendPlan& p, int64_t fit, int kv_heads, int32_t batch, const mvla_seq* seqs, bool counted, int32_t window, int32_t n_sink)
{
    int64_t keys = 0, longest = 1;
    for (int b = 0; b < batch; ++b) {
        if (seqs[b].n_q == 0) continue;
        const int64_t n = visible_keys(seqs[b], counted, window, n_sink);
        keys += n;
        longest = n > longest ? n : longest;
    }
    int64_t ctas = 0;
    const auto cut = [&](int cluster, int64_t part) {        // `part` keys to a CTA
        p.cluster = cluster;
        p.part_keys = part * cluster;
        p.splits = 1;
        p.blocks = 0;
        for (int b = 0; b < batch; ++b) {
            const int32_t n = parts_of(p, seqs[b], counted, window, n_sink);
            p.blocks += static_cast<int64_t>(n) * cluster;
            p.splits = n > p.splits ? n : p.splits;
        }
        ctas = p.blocks * kv_heads;
    };
    int64_t best = 0, best_cost = 0;
    int best_cluster = 1;
    for (int cluster = 1; cluster <= 8; cluster *= 2)
        for (int rounds = 0; rounds <= 4; ++rounds) {
            // (a cluster lies inside a group of multiprocessors, whose number need not divide)
            const int64_t at_once = fit - fit * (cluster == 1 ? 0 : cluster == 2 ? 3 : cluster == 4 ? 6 : 10) / 100;
            int64_t part = rounds ? (keys * kv_heads + rounds * at_once - 1) / (rounds * at_once) : (longest + cluster - 1) / cluster;
            part = std::max<int64_t>(part, (longest + 256 * cluster - 1) / (256 * cluster));
            part = std::max<int64_t>(64, (part + 63) / 64 * 64);
            cut(cluster, part);
            for (int tries = 0; rounds && ctas > rounds * at_once && part * cluster < longest && tries < 8; ++tries) cut(cluster, part += (part / 16 + 63) / 64 * 64);
            const int64_t mine = std::min(part, (longest + cluster - 1) / cluster);
            const int64_t cost = (ctas + at_once - 1) / at_once * (mine + 256) + (p.splits > 1 ? 128 + 4 * p.splits : 0) + (cluster > 1 ? 56 : 0);
            if (!best || cost < best_cost) { best = part; best_cost = cost; best_cluster = cluster; }
        }
    cut(best_cluster, best);
}

// Single tokens, of whose CTAs `ctas` fit on a multiprocessor.
inline AttendPlan plan_tokens(const ServeShape& c, int32_t batch, const mvla_seq* seqs, bool counted, int32_t window, int32_t n_sink, int ctas)
{
    AttendPlan p;
    p.form = kFormToken;
    p.rows = 0;
    for (int b = 0; b < batch; ++b) {
        p.total_q += seqs[b].n_q;
        p.total_kv += seqs[b].n_kv;
        p.rows = std::max(p.rows, static_cast<int32_t>(seqs[b].n_q * static_cast<int64_t>(c.n_heads / c.kv_heads)));
    }
    cut_page_tokens(p, static_cast<int64_t>(c.sm_count) * ctas, c.kv_heads, batch, seqs, counted, window, n_sink);
    if (p.splits > 1) {
        int64_t part_q = 0;
        for (int b = 0; b < batch; ++b) part_q += static_cast<int64_t>(parts_of(p, seqs[b], counted, window, n_sink)) * seqs[b].n_q;
        Workspace w;
        p.part_o = w.take(part_q * c.n_heads * c.head_dim * static_cast<int64_t>(sizeof(float)));
        p.part_ml = w.take(part_q * c.n_heads * 2 * static_cast<int64_t>(sizeof(float)));
        p.bytes = w.bytes;
    }
    return p;
}

// Blocks of queries by tiles of 128 rows, every sequence's keys cut into parts (clusters of 1, 2, 4 or 8 CTAs) of about the same length over the whole batch (a
// multiple of 64 keys to a CTA, at least 128), so that their CTAs fill whole rounds of those that fit: of one to four rounds, or no cut at all, what ends
// first.  In us: the tiles of its longest part and 4 for its start and end, `tile` each (with another CTA beside it); 1 and a 32nd of a head's elements where a cluster joins (with 1 alone 100
// queries of 32 heads of 128 had clusters of two, 11.8 us for 8.0); 5 for the kernel that joins parts, and what their sums, written and read, take at 6 TB/s.
constexpr double kTileUs = 1.3, kUnpackedTileUs = 2.2, kUnpackedPairUs = 1.7;
inline AttendPlan plan_page_tiles(const ServeShape& c, int32_t batch, const mvla_seq* seqs, bool counted, int32_t window, int32_t n_sink, int row_tiles, double tile)
{
    AttendPlan p;
    p.form = kFormPageTile;
    p.pack = pack_of(c.n_heads / c.kv_heads);
    p.queries = 128 / p.pack * row_tiles;
    const int64_t packs = c.n_heads / p.pack, each = c.head_dim <= 128 && row_tiles == 1 ? 2 : 1, slots = each * static_cast<int64_t>(c.sm_count);
    int64_t work = 0, longest = 1;
    const auto blocks_of = [&](const mvla_seq& s) { return (static_cast<int64_t>(s.n_q) + p.queries - 1) / p.queries; };
    for (int b = 0; b < batch; ++b) {
        p.total_q += seqs[b].n_q;
        p.total_kv += seqs[b].n_kv;
        if (seqs[b].n_q == 0) continue;
        const int64_t keys = visible_keys(seqs[b], counted, window, n_sink);
        work += blocks_of(seqs[b]) * packs * keys;
        longest = std::max(longest, keys);
    }
    int64_t ctas = 0, part_q = 0;
    const auto cut = [&](int cluster, int64_t part) {        // `part` keys to a CTA
        p.cluster = cluster;
        p.part_keys = part * cluster;
        p.blocks = part_q = 0;
        p.splits = 1;
        for (int b = 0; b < batch; ++b) {
            const int32_t n = parts_of(p, seqs[b], counted, window, n_sink);
            p.blocks += blocks_of(seqs[b]) * n;
            part_q += static_cast<int64_t>(seqs[b].n_q) * n;
            p.splits = std::max(p.splits, n);
        }
        ctas = p.blocks * packs * cluster;
    };
    int64_t best = 0;
    int best_cluster = 1;
    double best_cost = 0;
    for (int cluster = 1; cluster <= 8; cluster *= 2) {
        // (a cluster lies inside a group of multiprocessors, whose number need not divide)
        const int lost = cluster == 1 ? 0 : cluster == 2 ? 3 : cluster == 4 ? (each == 2 ? 6 : 11) : each == 2 ? 10 : 19;
        const int64_t at_once = slots - slots * lost / 100;
        for (int rounds = 0; rounds <= 4; ++rounds) {
            int64_t part = rounds ? (work + rounds * at_once - 1) / (rounds * at_once) : (longest + cluster - 1) / cluster;
            part = std::max<int64_t>({part, 128, (longest + 64 * cluster - 1) / (64 * cluster)});
            part = (part + 63) / 64 * 64;
            cut(cluster, part);
            for (int tries = 0; rounds && ctas > rounds * at_once && part * cluster < longest && tries < 16; ++tries) cut(cluster, part += std::max<int64_t>(64, part / 16 / 64 * 64));
            const double join = (cluster > 1 ? 1.0 + c.head_dim / 32.0 : 0.0) + (p.splits > 1 ? 5.0 + static_cast<double>(part_q) * c.n_heads * c.head_dim * 8 / 6e6 : 0.0);
            const int64_t mine = (std::min(part, (longest + cluster - 1) / cluster) + 63) / 64;
            const double cost = static_cast<double>((ctas + at_once - 1) / at_once) * static_cast<double>(mine + 4) * tile + join;
            if (!best || cost < best_cost) { best = part; best_cost = cost; best_cluster = cluster; }
        }
    }
    cut(best_cluster, best);
    if (p.splits > 1) {
        Workspace w;
        p.part_o = w.take(part_q * c.n_heads * c.head_dim * static_cast<int64_t>(sizeof(float)));
        p.part_ml = w.take(part_q * c.n_heads * 2 * static_cast<int64_t>(sizeof(float)));
        p.bytes = w.bytes;
    }
    return p;
}

// Few query rows to a key head: the token form unpacks quantised rows as it reads them, where the tile form has them unpacked first.  Rows of their own type: the tile form's
// larger copies win over long sequences, although its rows are mostly empty; its start and end take 3 to 10 us longer.  `keys`: of the batch, `mean`: of a sequence.  us, token / tile
// form.  Heads of 64, 32 over 8: one token over 1000 rows 6.3 / 10.2, over 60000 35 / 35, 64 requests over 500 to 1500 39 / 53; four tokens over 1000 7.2 / 10.4, over 8000 15.5 / 15.2, 64 requests 48 / 52.  Of
// 96, 16 heads: one token over 60000 rows 82 / 79, 16 requests over 1300 to 4000 66 / 72.  Of 128, 32 over 8: one token over 1000 7.7 / 12.8, over 8000 16.7 / 15.5, over 60000
// 63 / 50, 64 requests over 170 to 500 33 / 34, 16 over 1300 to 4000 49 / 44; four tokens over 1000 9.6 / 13.0, four requests over 500 to 1500 13.7 / 15.9, 16 29.7 / 26.8.  Of 256,
// 32 over 8: one token over 1000 10.4 / 18.4, 16 requests over 500 to 1500 54 / 46, 64 over 170 to 500 78 / 76; 16 over 2, over 8000 24 / 19.
inline bool page_by_tokens(int kind, int head_dim, int64_t rows, int64_t keys, int64_t mean, int kv_heads)
{
    if (rows > kTokenRows) return false;
    if (kind != MVLA_PAGE_ROWS) return true;
    const int64_t all = keys * kv_heads;
    if (rows > 8) return head_dim <= 64 ? mean <= 4096 : head_dim <= 192 && mean <= 1280 && all <= 40960;
    return head_dim <= 96 || mean <= (head_dim <= 192 ? 1280 : 512) || (all <= 32768 && (head_dim <= 192 || mean <= 1280));
}

// Tiles of query rows that share what is unpacked on the way, 0: unpacked first.  Unpacking first costs 0.15 us for 1000 rows of a head (their bytes, twice) and a kernel's start, on the
// way every CTA does it for one tile of rows or two (heads of up to 128 elements).  `keys`: of the batch, `mean`: of a sequence.  us, on the way / first, 32 heads in groups of 4, e4m3: 5 tokens
// over 60000 rows (one tile) 63 / 119; 4 chunks of 56 over 3100 to 5500 (two) 49 / 58, of 33 over 4000 (two) 40 / 49, 16 of 60 over 400 to 800 34.5 / 34.2, one over 4000 29 / 26, over 9000 36 / 37;
// 100 over 4096 (four) 34 / 28; 512 over 8192 (16) 123 / 94.  16 heads of 64: 200 over 4000 (two) 25.4 / 24.7, over 30000 89 / 102.
inline int32_t unpacked_row_tiles(const ServeShape& c, int32_t batch, const mvla_seq* seqs, int64_t keys, int64_t mean)
{
    const int64_t queries = 128 / pack_of(c.n_heads / c.kv_heads);
    int64_t most = 0;
    for (int b = 0; b < batch; ++b) most = std::max(most, (static_cast<int64_t>(seqs[b].n_q) + queries - 1) / queries);
    if (most <= 1) return 1;
    return most > 2 || mean < 2048 || keys * c.kv_heads <= 65536 ? 0 : c.head_dim <= 128 ? 2 : 1;
}

// fp32: blocks of 8 query rows, every sequence's keys cut into as many parts, 64 at most: of all such cuts the one that ends first, in rounds of a CTA's warps over 16 keys
// each (2 us): those of its longest part and 1.5 for its start and end, for every round of the CTAs that fit, and 2 for the kernel that joins parts (one token over 2000 rows of 8 heads
// of 64: 7 parts of three rounds 12.5 us, 16 of one 8.0; over 300 rows of heads of 128 one part 14.5, five 8.0).
inline AttendPlan plan_page_fma(const ServeShape& c, int32_t batch, const mvla_seq* seqs, bool counted, int32_t window, int32_t n_sink)
{
    AttendPlan p;
    p.rows = 8;
    int64_t longest = 0;
    for (int b = 0; b < batch; ++b) {
        p.total_q += seqs[b].n_q;
        p.total_kv += seqs[b].n_kv;
        p.blocks += (static_cast<int64_t>(seqs[b].n_q) * (c.n_heads / c.kv_heads) + 7) / 8;
        if (seqs[b].n_q) longest = std::max(longest, visible_keys(seqs[b], counted, window, n_sink));
    }
    const int64_t slots = static_cast<int64_t>(c.sm_count) * page_fma_ctas(c.head_dim / 32), keys = 16 * page_fma_warps(c.head_dim / 32);
    double best = 0;
    for (int64_t n = 1; n <= 64; ++n) {
        const int64_t part = (longest + n - 1) / n;
        const double cost = static_cast<double>((p.blocks * c.kv_heads * n + slots - 1) / slots) * (static_cast<double>((part + keys - 1) / keys) + 1.5) + (n > 1 ? 2 : 0);
        if (n == 1 || cost < best) { best = cost; p.splits = static_cast<int32_t>(n); }
    }
    if (p.splits > 1) {
        Workspace w;
        p.part_o = w.take(p.total_q * p.splits * c.n_heads * c.head_dim * static_cast<int64_t>(sizeof(float)));
        p.part_ml = w.take(p.total_q * p.splits * c.n_heads * 2 * static_cast<int64_t>(sizeof(float)));
        p.bytes = w.bytes;
    }
    return p;
}

inline PageAttendPlan plan_page_attention(const ServeShape& v, int32_t batch, const mvla_seq* seqs, const mvla_paged_attention* a)
{
    PageAttendPlan p;
    const ServeShape h = hidden_shape(v);
    const bool counted = !a->kv_len;
    int64_t most_rows = 0;
    for (int b = 0; b < batch; ++b) most_rows = std::max(most_rows, seqs[b].n_q * static_cast<int64_t>(v.n_heads / v.kv_heads));
    int64_t keys = 0, active = 0;
    for (int b = 0; b < batch; ++b) {
        if (seqs[b].n_q == 0) continue;
        keys += visible_keys(seqs[b], counted, a->window, a->n_sink);
        ++active;
    }
    const int64_t mean = keys / std::max<int64_t>(active, 1);
    const bool tokens = h.dtype != MVLA_DTYPE_FP32 && page_by_tokens(a->pages.kind, v.head_dim, most_rows, keys, mean, v.kv_heads);
    if (h.dtype != MVLA_DTYPE_FP32 && a->pages.kind != MVLA_PAGE_ROWS && !tokens) p.unpack = unpacked_row_tiles(h, batch, seqs, keys, mean);
    p.attend = h.dtype == MVLA_DTYPE_FP32 ? plan_page_fma(h, batch, seqs, counted, a->window, a->n_sink)
             : tokens ? plan_tokens(h, batch, seqs, counted, a->window, a->n_sink, page_token_ctas(a->pages.kind, v.head_dim / 32, most_rows <= 8 ? 1 : 2))
                      : plan_page_tiles(h, batch, seqs, counted, a->window, a->n_sink, p.unpack == 2 ? 2 : 1, p.unpack == 2 ? kUnpackedPairUs : p.unpack ? kUnpackedTileUs : kTileUs);
    p.bytes = p.attend.bytes;
    if (a->pages.kind == MVLA_PAGE_ROWS || tokens || p.unpack) return p;
    Workspace w;
    w.take(p.attend.bytes);
    for (int b = 0; b < batch; ++b) p.dense_tiles += seen_tiles(seqs[b], a->window, a->n_sink);
    const int64_t bytes = p.dense_tiles * kPageTile * v.kv_heads * v.head_dim * static_cast<int64_t>(v.wide);
    p.dense_k = w.take(bytes);
    p.dense_v = w.take(bytes);
    p.bytes = w.bytes;
    return p;
}

// Pointers of a call that has queries.
inline int32_t check_page_attention_memory(const ServeShape& v, int32_t batch, const mvla_paged_attention* a, const PageAttendPlan& plan)
{
    Range pool[4];
    const int32_t rc = check_pool(v, a->pages, pool);
    if (rc != MVLA_OK) return rc;
    if (!a->q || !a->out || (plan.attend.total_kv > 0 && !a->table)) return MVLA_ERR_INVALID_ARG;
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->lse, 4) || !aligned(a->table, 4) || !aligned(a->kv_len, 4) || !aligned(a->workspace, 256))
        return MVLA_ERR_INVALID_ARG;
    if (plan.bytes > 0 && (!a->workspace || a->workspace_bytes < plan.bytes)) return MVLA_ERR_INVALID_ARG;
    const int64_t qw = static_cast<int64_t>(v.n_heads) * v.head_dim * static_cast<int64_t>(v.wide);
    const Range in[7] = {range_of(a->q, a->q_rows * qw), table_range(batch, a->table, a->table_stride), range_of(a->kv_len, batch * 4), pool[0], pool[1], pool[2], pool[3]};
    const Range out[3] = {range_of(a->out, a->q_rows * qw), range_of(a->lse, a->q_rows * v.n_heads * 4), range_of(plan.bytes ? a->workspace : nullptr, plan.bytes)};
    for (int i = 0; i < 3; ++i) {
        for (const Range& r : in) if (meet(out[i], r)) return MVLA_ERR_INVALID_ARG;
        for (int j = i + 1; j < 3; ++j) if (meet(out[i], out[j])) return MVLA_ERR_INVALID_ARG;
    }
    return MVLA_OK;
}

}  // namespace mvla
