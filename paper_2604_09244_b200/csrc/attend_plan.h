// Host arithmetic of a windowed-attention call: its blocks, how the visible keys are split, and where its workspace lies.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "mvla_prune.h"

namespace mvla {

// Token form (attend_token.cu): subtiles of 16 keys in a warp's tile; shared memory of a CTA, four warps with three tiles each, in whole groups of 64
// columns of the values; and the CTAs that fit on a multiprocessor (four at most: by registers).
constexpr int token_sub(int pieces_of_32) { return pieces_of_32 <= 2 ? 2 : 1; }
constexpr int token_smem(int pieces_of_32, int elem)
{
    return 4 * 3 * token_sub(pieces_of_32) * (2 * pieces_of_32 + 4 * ((pieces_of_32 + 1) / 2)) * 32 * 8 * elem;
}
constexpr int token_ctas(int pieces_of_32, int elem)
{
    const int n = 220 * 1024 / (token_smem(pieces_of_32, elem) + 8 * 1024);
    return n > 4 ? 4 : n < 1 ? 1 : n;
}

// What the plans and checks of a call go by in its context.
struct ServeShape {
    int dtype, hidden_dtype;            // MVLA_DTYPE_* of q / k / v and of the rows beside them (bf16 where q / k / v are e4m3)
    int n_heads, kv_heads, head_dim, max_batch, sm_count;
    size_t elem, wide;                  // bytes per element of q / k / v, and of the rows beside them
};

// What a call reads of a sequence at most, by its descriptor (positions that are data may leave anything visible).
inline int64_t visible_keys(const mvla_seq& s, bool counted, int32_t window, int32_t n_sink)
{
    if (!counted) return s.n_kv;
    const int64_t all = static_cast<int64_t>(window) + s.n_q - 1 + n_sink;
    return all < s.n_kv ? all : s.n_kv;
}

struct Workspace {
    int64_t bytes = 0;
    int64_t take(int64_t n)
    {
        const int64_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};

constexpr int kMaxTiles = 2048;          // tiles of keys that a CTA of the tile kernels walks (its list of them: 11 bits an entry)

// kFormFma: by FMAs.  kFormTile: by tiles of 128 query rows on the tensor cores (e4m3: after widening to fp16).
// kFormToken: at most 16 query rows to a key head, straight from global memory.
enum AttendForm { kFormFma, kFormTile, kFormToken };

// A sequence of at most so many query rows to a key head counts as single tokens: its bf16 weights keep what rounding leaves of them, in the token form and
// in the tile form, so that the form that its batch is given costs no bits.
constexpr int kTokenRows = 16;

// Few query rows to a key head: the token form reads e4m3 rows as they are and keeps scores for the weights, where the tile form widens all rows and
// goes over the keys a second time; heads of 64 are tiles too small for it.  Else the tile form's larger copies win although its rows are mostly
// empty, but for calls too short to fill the device with its parts of four tiles and more, of up to eight rows (beyond, the token form does all twice).
// us, token / tile form, one token where nothing else is said: e4m3, 60000 rows of 8 heads of 128 44 / 129; with weights, 800 rows 11.7 / 22.6; heads of
// 64, 60000 rows of 8 35.4 / 37.0.  bf16 without weights, 4 query heads to each of 8 heads of 128, 800 / 4000 / 16000 / 131071 rows 8.5 / 12.8,
// 12.4 / 14.2, 23.4 / 21.4, 107 / 89; 32 heads of 128 with a query head each 11.0 / 15.2, 20.7 / 24.8, 57 / 53, 394 / 331; 32 of 96 10.3 / 13.8, 18.0 / 19.9,
// 46 / 46, 310 / 287; 16 of 256 12.9 / 17.5, 23.1 / 25.3, 58 / 57, 399 / 357; 2, 3 and 4 tokens (8, 12, 16 rows) over 200 rows 9.7 / 9.8, 12.1 / 9.8, 14.5 / 9.8,
// over 30000 36 / 31, 41 / 31, 43 / 31; 32 requests over 700 to 800 rows 28.2 / 26.5.  The tile form cuts all sequences into as many parts, so lengths
// have to be alike, the longest half as long again as the average at most (16 requests over 8 heads: 1500 to 3000 rows 45.1 / 40.0, 500 to 4000 46.1 / 45.4,
// 500 to 60000 381 / 505, 100 to 131071 794 / 1095).
inline bool by_tokens(int dtype, int head_dim, int64_t rows, bool mass, bool alike, int64_t all_keys)
{
    return rows <= kTokenRows && (dtype == MVLA_DTYPE_FP8_E4M3 || mass || head_dim <= 64 || !alike || (rows <= 8 && all_keys < 8192));
}

struct AttendPlan {
    AttendForm form = kFormFma;
    int32_t rows = 32;           // query rows of a block (a block shares a key head: queries x heads of a group)
    int32_t pack = 1;            // heads side by side in a tile of rows
    int32_t queries = 0;         // queries of a block of the tile form
    int32_t splits = 1, mass_parts = 1;
    int64_t total_q = 0, total_kv = 0, blocks = 0;
    // offsets in the workspace, -1: not used
    int64_t part_o = -1, part_ml = -1, lse2 = -1, part_mass = -1, wide_q = -1, wide_k = -1, wide_v = -1, logits = -1, bytes = 0;
    int64_t part_keys = 0;       // single tokens: keys of a part
    int64_t logit_floats = 0;
};

// Parts that a sequence's visible keys are cut into.
inline int32_t parts_of(const AttendPlan& p, const mvla_seq& s, bool counted, int32_t window, int32_t n_sink)
{
    if (s.n_q == 0) return 0;
    if (p.form != kFormToken) return p.splits;
    const int64_t n = (visible_keys(s, counted, window, n_sink) + p.part_keys - 1) / p.part_keys;
    return n < 1 ? 1 : static_cast<int32_t>(n);
}

// Heads of a group that share a tile of 128 rows: as many as divide the group, 32 at most.
inline int pack_of(int group)
{
    int p = group < 32 ? group : 32;
    while (group % p) --p;
    return p;
}

inline AttendPlan plan_attend(const ServeShape& c, int32_t batch, const mvla_seq* seqs, bool counted, int32_t window, int32_t n_sink, bool mass)
{
    AttendPlan p;
    const int group = c.n_heads / c.kv_heads;
    int64_t longest = 0, longest_kv = 0, most_rows = 0, all_keys = 0, active = 0;
    for (int b = 0; b < batch; ++b) {
        const mvla_seq& s = seqs[b];
        p.total_q += s.n_q;
        p.total_kv += s.n_kv;
        if (s.n_q == 0) continue;
        const int64_t keys = visible_keys(s, counted, window, n_sink), rows = static_cast<int64_t>(s.n_q) * group;
        longest = keys > longest ? keys : longest;
        all_keys += keys;
        ++active;
        longest_kv = s.n_kv > longest_kv ? s.n_kv : longest_kv;
        most_rows = rows > most_rows ? rows : most_rows;
    }
    if (c.dtype == MVLA_DTYPE_FP32) {
        // (four tokens over 200 to 900 rows 20.6 us with blocks of 8 rows, 28.7 with 32; 30000 rows of 8 heads 81 and 94)
        p.rows = most_rows <= 8 ? 8 : 32;
        int64_t row_blocks = 0, key_tiles = 0;
        for (int b = 0; b < batch; ++b) {
            p.blocks += (static_cast<int64_t>(seqs[b].n_q) * group + p.rows - 1) / p.rows;
            row_blocks += (static_cast<int64_t>(seqs[b].n_q) * group + 31) / 32;
            key_tiles += (static_cast<int64_t>(seqs[b].n_kv) + 63) / 64;
        }
        // weights: enough CTAs (64 keys of a head each) for every multiprocessor eight times, since the first keys have the most rows to
        // go through, of at least two blocks of 32 rows on average
        int64_t runs = key_tiles == 0 ? 1 : 8 * static_cast<int64_t>(c.sm_count) / (key_tiles * c.kv_heads);
        runs = runs > row_blocks / 2 ? row_blocks / 2 : runs;
        p.mass_parts = static_cast<int32_t>(c.kv_heads * (runs < 1 ? 1 : runs));
        if (p.blocks > 0) {
            // enough CTAs for every multiprocessor twice, of at least four tiles of 64 keys
            const int64_t ctas = p.blocks * c.kv_heads;
            int64_t n = (2 * static_cast<int64_t>(c.sm_count) + ctas - 1) / ctas;
            const int64_t most = longest / 256;
            n = n > most ? most : n;
            n = n > 64 ? 64 : n;
            p.splits = n < 1 ? 1 : static_cast<int32_t>(n);
        }
    } else if (by_tokens(c.dtype, c.head_dim, most_rows, mass, 2 * longest * active <= 3 * all_keys, all_keys)) {
        // Parts of equal length over the whole batch, a multiple of 64 keys (a tile for each warp), so that their CTAs fill whole rounds of
        // those that fit: of one to four rounds the ones that end first, by the keys of a round's longest part and 128 for its start
        // and end.  256 parts to a sequence at most (the join reads them all).
        p.form = kFormToken;
        p.rows = static_cast<int32_t>(most_rows);
        int64_t keys = 0;
        for (int b = 0; b < batch; ++b) {
            if (seqs[b].n_q == 0) continue;
            keys += visible_keys(seqs[b], counted, window, n_sink);
            p.logit_floats += mass ? static_cast<int64_t>(seqs[b].n_q) * c.n_heads * seqs[b].n_kv : 0;
        }
        const int64_t fit = static_cast<int64_t>(c.sm_count) * token_ctas(c.head_dim / 32, static_cast<int>(c.elem));
        const auto ctas_of = [&](int64_t part) {
            int64_t n = 0;
            p.part_keys = part;
            for (int b = 0; b < batch; ++b) n += parts_of(p, seqs[b], counted, window, n_sink);
            return n * c.kv_heads;
        };
        int64_t best = 0, best_cost = 0;
        for (int rounds = 1; rounds <= 4; ++rounds) {
            int64_t part = (keys * c.kv_heads + rounds * fit - 1) / (rounds * fit);
            part = part < (longest + 255) / 256 ? (longest + 255) / 256 : part;
            part = part < 64 ? 64 : (part + 63) / 64 * 64;
            int64_t n = ctas_of(part);
            for (int tries = 0; n > rounds * fit && tries < 8; ++tries) {
                part += (part / 16 + 63) / 64 * 64;
                n = ctas_of(part);
            }
            const int64_t cost = (n + fit - 1) / fit * ((part < longest ? part : longest) + 128);
            if (!best || cost < best_cost) { best = part; best_cost = cost; }
        }
        p.part_keys = best;
        for (int b = 0; b < batch; ++b) {
            const int32_t n = parts_of(p, seqs[b], counted, window, n_sink);
            p.blocks += n;
            p.splits = n > p.splits ? n : p.splits;
        }
    } else {
        p.form = kFormTile;
        p.pack = pack_of(group);
        const int per = 128 / p.pack;
        const int64_t tile = 64;                             // keys (attend_tile.cu)
        p.queries = per;
        int64_t most_q = 0;
        for (int b = 0; b < batch; ++b) {
            p.blocks += (static_cast<int64_t>(seqs[b].n_q) + p.queries - 1) / p.queries;
            most_q = seqs[b].n_q > most_q ? seqs[b].n_q : most_q;
        }
        const int64_t packs = c.n_heads / p.pack;
        if (p.blocks > 0) {
            // one round of the CTAs that fit; parts of at least four tiles; and no more tiles than a CTA's list holds
            const int64_t ctas = p.blocks * packs, tiles = (longest + tile - 1) / tile;
            int64_t n = (c.head_dim <= 128 ? 2 : 1) * static_cast<int64_t>(c.sm_count) / ctas;
            const int64_t most = tiles / 4, least = ((longest_kv + tile - 1) / tile + kMaxTiles - 1) / kMaxTiles;
            n = n > most ? most : n;
            n = n > 64 ? 64 : n;
            n = n < least ? least : n;
            p.splits = n < 1 ? 1 : static_cast<int32_t>(n);
        }
        const int64_t runs = ((most_q + per - 1) / per + kMaxTiles - 1) / kMaxTiles;
        p.mass_parts = static_cast<int32_t>(packs * (runs < 1 ? 1 : runs));
    }
    Workspace w;
    const int64_t qh = p.total_q * c.n_heads;
    if (p.splits > 1 || (mass && p.form == kFormToken)) {
        int64_t part_q = 0;
        for (int b = 0; b < batch; ++b) part_q += static_cast<int64_t>(parts_of(p, seqs[b], counted, window, n_sink)) * seqs[b].n_q;
        if (p.splits > 1) p.part_o = w.take(part_q * c.n_heads * c.head_dim * static_cast<int64_t>(sizeof(float)));
        p.part_ml = w.take(part_q * c.n_heads * 2 * static_cast<int64_t>(sizeof(float)));
    }
    if (mass) {
        if (p.form != kFormToken) p.lse2 = w.take(qh * static_cast<int64_t>(sizeof(float)));
        if (p.form == kFormToken) p.logits = w.take(p.logit_floats * static_cast<int64_t>(sizeof(float)));
        else p.part_mass = w.take(p.mass_parts * p.total_kv * static_cast<int64_t>(sizeof(float)));
    }
    if (p.form == kFormTile && c.dtype == MVLA_DTYPE_FP8_E4M3) {
        p.wide_q = w.take(qh * c.head_dim * 2);
        p.wide_k = w.take(p.total_kv * c.kv_heads * c.head_dim * 2);
        p.wide_v = w.take(p.total_kv * c.kv_heads * c.head_dim * 2);
    }
    p.bytes = w.bytes;
    return p;
}

}  // namespace mvla
