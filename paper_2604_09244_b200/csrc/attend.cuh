// Device side of the windowed attention that its kernels share: who sees whom, and which tiles of keys a block of queries visits.
#pragma once

#include "device_utils.cuh"
#include "serve.h"

#include <cuda_fp8.h>

namespace mvla {

// Weights that meet the values in fp16 are counted in units of 2^-kF16Lift of their row's reference: none lies more than 2^8 above the reference, so that
// the largest is 2^15 and fits, and one stays a normal number (11 bits) down to 2^-21 of the reference instead of 2^-14, and is nothing below 2^-32
// instead of 2^-25.  The sum that divides them is taken of the same units, and the reference that is handed on is less by as much.
constexpr float kF16Lift = 7.f;

__device__ __forceinline__ int seq_len(const AttArgs& a, const AttSeq& s)
{
    return a.kv_len ? min(max(a.kv_len[s.index], 0), s.n_kv) : s.n_kv;
}
// (all negative positions see the same, nothing: one of them will do)
__device__ __forceinline__ int query_pos(const AttArgs& a, const AttSeq& s, int len, int i)
{
    return max(a.q_pos ? a.q_pos[s.q_row + i] : len - s.n_q + i, -1);
}
// Position of row j of a sequence, -1 where nobody sees it.
__device__ __forceinline__ int key_pos(const AttArgs& a, const AttSeq& s, int len, int j)
{
    return j >= len ? -1 : a.kv_pos ? a.kv_pos[s.kv_row + j] : j;
}
// (p - c cannot overflow: c is not negative and not above p where it is taken)
__device__ __forceinline__ bool sees(int p, int c, int window, int n_sink)
{
    return c >= 0 && c <= p && (p - c < window || c < n_sink);
}
// Whether some query with a position in [lo, hi] may see a key at c.
__device__ __forceinline__ bool some_sees(int lo, int hi, int c, int window, int n_sink)
{
    return c >= 0 && c <= hi && (c >= lo || lo - c < window || c < n_sink);
}
// The last sequence whose field (ascending over the batch) is not above x: by halves, since every look costs a constant load's latency.
template <class Field>
__device__ __forceinline__ int seq_at(const AttArgs& a, int x, Field field)
{
    int lo = 0, n = a.n_seq;
    while (n > 1) {
        const int half = n >> 1;
        if (field(a.s[lo + half]) <= x) lo += half;
        n -= half;
    }
    return lo;
}
// The block of the launch's grid that `blk` is: its sequence.
__device__ __forceinline__ int seq_of_block(const AttArgs& a, int blk) { return seq_at(a, blk, [](const AttSeq& s) { return s.blk0; }); }
__device__ __forceinline__ int seq_of_query(const AttArgs& a, int qp) { return seq_at(a, qp, [](const AttSeq& s) { return s.qp0; }); }
__device__ __forceinline__ int seq_of_key(const AttArgs& a, int kvp) { return seq_at(a, kvp, [](const AttSeq& s) { return s.kvp0; }); }
// Tiles of `tile` keys that queries at [lo, hi] may see: `sinks` tiles from the first on, then those from `first` on, `count` in all.
// Where the positions are data every tile of the sequence is named, and looked at when it comes up.
struct TileRange {
    int sinks, first, count;
    __device__ __forceinline__ int tile(int t) const { return t < sinks ? t : first + t - sinks; }
};
__device__ __forceinline__ TileRange counted_tiles(int len, int lo, int hi, int tile, int window, int n_sink)
{
    TileRange r = {0, 0, 0};
    const int n = (min(len - 1, max(hi, -1)) + 1 + tile - 1) / tile;     // (hi may be the last position of its type)
    r.first = min((window > lo ? 0 : lo - window + 1) / tile, n);
    r.sinks = min(static_cast<int>((static_cast<int64_t>(n_sink) + tile - 1) / tile), r.first);
    r.count = r.sinks + n - r.first;
    return r;
}
__device__ __forceinline__ TileRange tile_range(const AttArgs& a, int len, int lo, int hi, int tile)
{
    if (!a.kv_pos) return counted_tiles(len, lo, hi, tile, a.window, a.n_sink);
    const int n = (len + tile - 1) / tile;
    return {0, 0, n};
}

}  // namespace mvla
