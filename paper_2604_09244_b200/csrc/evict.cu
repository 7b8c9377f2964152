// Eviction from a cache by accumulated attention weight: which rows stay, and the moves that leave them in front.
//
// Kept rows that lie below the new length stay where they are; those behind it move into the holes.  Sources and
// destinations are then different rows by construction, so all moves may run at once and in place, and a decode step that is one row
// over its budget moves one row instead of the cache.
//
// evict_select_kernel: a cluster of one to eight CTAs a sequence, by its length; a CTA has a run of its rows.  Every row has a 32-bit key
// (its weight's bits in order of size; protected rows above all, hidden rows below all); three rounds of 2048-bin counts over the keys, most
// significant bits first (sign, exponent and two bits of the fraction, so that weights of one size spread over bins), give the key of the
// last row that stays and how many of its equals do.  A round looks for its bin in two steps, sums of 64 bins and then the 64 of one sum, so
// that little is read out of the other CTAs' shared memory; every CTA does so for itself.  Then every warp walks a run of rows in
// ascending order and counts, keeps a bit for each row that stays, and goes over the bits once more to write.
// Keys are kept in shared memory where they fit.  Bound by the latency of its passes: a barrier of the cluster is about 0.8 us.
// evict_move_kernel: one warp a 2 KB piece of a moved row.  Bound by bytes.
//
// B200: 16 sequences one row over their budgets (one kernel) 8.3 us; 16 of 784 to 832 rows of 32 + 32 heads of 128 cut to three tenths 25 us, of it
// 16 the move's 88 MB; 65537 rows of 8 + 8 heads cut to an eighth 37 us, of it 11 the move (with one CTA 300; reading all bins of all
// CTAs, and taking the keys apart again for the second walk, 46).  Equal bins of a warp counted together: 54 (the atomics are not what it waits for).
// The selection's 25 us of the last: seven barriers of the cluster are a quarter, the rest is eight multiprocessors going over 8192 rows each six times.
#include "device_utils.cuh"
#include "serve.h"

#include <algorithm>

namespace mvla {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kKeysInSmem = 49152;           // 192 KB
// From here on a sequence gets another CTA, up to kMaxCluster.  us with 2048 / 4096 / 8192: 3000 rows 15.8 / 12.9 / 12.9, 6000 17.1 / 18.7 / 17.3,
// 12000 19.7 / 20.8 / 25.2, 30000 30.1 / 29.9 / 36.0.
constexpr int kRowsPerCta = 4096;
constexpr int kBins = 2 * kThreads;          // of a round: eleven bits of the key
constexpr int kMoveThreads = 256;
constexpr int kPiece = 2048;
constexpr int kMovesInSelect = 4;            // rows that the selecting CTA moves itself (16 sequences one row over: 8.6 us, by a second kernel 10.6)

__device__ __forceinline__ int seq_rows(const EvictArgs& a, const EvictSeq& s)
{
    return a.kv_len ? min(max(a.kv_len[s.index], 0), s.n_kv) : s.n_kv;
}
// Key of a row at position c whose weight is w; `last`: the largest position of its sequence.
__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, int c, float w, int last)
{
    if (c < 0) return 0u;
    if (c < a.n_sink || last - c < a.n_recent) return 0xFFFFFFFFu;
    if (w != w) return 1u;                                    // NaN: below every number
    const uint32_t u = __float_as_uint(w + 0.f);              // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;            // (from 0x007FFFFF, -infinity, to 0xFF800000, +infinity)
}
// A 2 KB piece of a row, or what is left of it (16-byte steps).
__device__ __forceinline__ void move_piece(char* dst, const char* src, int bytes, int lane)
{
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((i * 32 + lane) * 16 < bytes) x[i] = *reinterpret_cast<const uint4*>(src + (i * 32 + lane) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((i * 32 + lane) * 16 < bytes) *reinterpret_cast<uint4*>(dst + (i * 32 + lane) * 16) = x[i];
}
// Largest over the block, in every thread.
__device__ __forceinline__ int block_max(int v, int* red)
{
    v = __reduce_max_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, red[threadIdx.x & 31]);
}
__device__ __forceinline__ int ld_peer(const int* p, uint32_t rank)
{
    uint32_t at;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ int2 ld_peer2(const int* p, uint32_t rank)
{
    uint32_t at;
    int2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync()
{
    cluster_arrive_release();
    cluster_wait_acquire();
}
// Inclusive sum over the lanes.
__device__ __forceinline__ int sum_upto(int x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// Exclusive sum over the CTA's warps of one value per warp (the same in all its lanes), and the total.
__device__ __forceinline__ int warps_before(int v, int* red, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    const int mine = red[lane], x = sum_upto(mine);
    *total = __shfl_sync(0xffffffffu, x, 31);
    return __shfl_sync(0xffffffffu, x - mine, warp);
}

__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ EvictArgs a)
{
    extern __shared__ uint32_t cached[];
    __shared__ __align__(8) int hist[2][kBins];
    __shared__ int red[kWarps];
    __shared__ __align__(8) int slots[4];
    __shared__ int coarse[2][kWarps], found[2];
    uint32_t n_ranks;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ranks));
    const uint32_t rank = cluster_ctarank();
    const int seq = static_cast<int>(blockIdx.x / n_ranks);
    const EvictSeq& s = a.s[seq];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    pdl_wait();
    const int n = seq_rows(a, s), m = min(n, s.budget);
    const int64_t row = s.kv_row;
    __syncthreads();                                          // (kv_len_out may be kv_len: everybody of the CTA has read it)
    // this CTA's rows: whole runs of 1024
    const int per_rank = ((n + static_cast<int>(n_ranks) - 1) / static_cast<int>(n_ranks) + kThreads - 1) / kThreads * kThreads;
    const int r0 = min(static_cast<int>(rank) * per_rank, n), r1 = min(r0 + per_rank, n);
    if (m == n || m == 0) {                                   // everything stays, or nothing
        const int end = min(r1, m);
        if (a.pos_out != a.pos) for (int j = r0 + t; j < end; j += kThreads) a.pos_out[row + j] = a.pos[row + j];
        if (a.mass_out != a.mass) for (int j = r0 + t; j < end; j += kThreads) a.mass_out[row + j] = a.mass[row + j];
        if (a.kept_idx) for (int j = r0 + t; j < end; j += kThreads) a.kept_idx[row + j] = j;
        if (t == 0 && rank == 0) {
            a.n_moves[seq] = 0;
            if (a.kv_len_out) a.kv_len_out[s.index] = m;      // (another CTA of the cluster that reads it now ends here just the same)
        }
        return;
    }
    const bool fits = r1 - r0 <= kKeysInSmem;
    int last = -1;
#pragma unroll 4
    for (int j = r0 + t; j < r1; j += kThreads) {             // (the weights on their way together with the positions)
        last = max(last, a.pos[row + j]);
        if (fits) cached[j - r0] = __float_as_uint(a.mass[row + j]);
    }
    last = block_max(last, red);
    hist[0][t] = hist[0][t + kThreads] = 0;
    if (n_ranks > 1) {
        if (t == 0) slots[0] = last;
        cluster_sync();
        last = __reduce_max_sync(0xffffffffu, lane < static_cast<int>(n_ranks) ? ld_peer(&slots[0], lane) : -1);
    }
    const auto key_at = [&](int j) { return fits ? cached[j - r0] : key_of(a, a.pos[row + j], a.mass[row + j], last); };
    if (fits) {
#pragma unroll 4
        for (int j = r0 + t; j < r1; j += kThreads) cached[j - r0] = key_of(a, a.pos[row + j], __uint_as_float(cached[j - r0]), last);
    }
    // The key of the m-th row in descending order, eleven, eleven and ten bits; `left`: rows still to be found among those with the bits so far.
    uint32_t prefix = 0;
    int left = m, equal_here = 0, equal_before = 0;          // rows with that key: in this CTA, in the CTAs before it
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
        int* const mine = hist[round & 1];
        const uint32_t above = round == 0 ? 0u : round == 1 ? 0xFFE00000u : 0xFFFFFC00u, bins = round < 2 ? 2047u : 1023u;
        __syncthreads();
#pragma unroll 2
        for (int j = r0 + t; j < r1; j += kThreads) {
            const uint32_t k = key_at(j);
            if ((k & above) == prefix) atomicAdd(&mine[(k >> shift) & bins], 1);
        }
        __syncthreads();
        {                                                     // 64 bins a warp
            const int2 c = *reinterpret_cast<const int2*>(&mine[64 * warp + 2 * lane]);
            const int sum = __reduce_add_sync(0xffffffffu, c.x + c.y);
            if (lane == 0) coarse[round & 1][warp] = sum;
        }
        if (n_ranks > 1) cluster_sync();
        else __syncthreads();
        // (the other buffer was read by everybody before this barrier)
        hist[(round + 1) & 1][t] = hist[(round + 1) & 1][t + kThreads] = 0;
        if (warp == 0) {
            // from the top: the 64 bins among which the row is found, then the bin; the cluster's counts all on their way at once
            int c = 0;
#pragma unroll
            for (uint32_t i = 0; i < kMaxCluster; ++i) c += i < n_ranks ? ld_peer(&coarse[round & 1][31 - lane], (i + rank) & (n_ranks - 1)) : 0;
            int upto = sum_upto(c);
            unsigned hit = __ballot_sync(0xffffffffu, upto >= left) | 1u << 31;
            const int at = __ffs(hit) - 1, base = 64 * (31 - at);
            left -= __shfl_sync(0xffffffffu, upto - c, at);
            int c0 = 0, c1 = 0;
#pragma unroll
            for (uint32_t i = 0; i < kMaxCluster; ++i) {
                const int2 x = i < n_ranks ? ld_peer2(&mine[base + 62 - 2 * lane], (i + rank) & (n_ranks - 1)) : make_int2(0, 0);
                c0 += x.y;
                c1 += x.x;
            }
            upto = sum_upto(c0 + c1);
            hit = __ballot_sync(0xffffffffu, upto >= left) | 1u << 31;
            if (lane == __ffs(hit) - 1) {
                const int rest = left - (upto - c0 - c1);
                const bool second = rest > c0;
                found[0] = base + 63 - 2 * lane - (second ? 1 : 0);
                found[1] = rest - (second ? c0 : 0);
            }
        }
        __syncthreads();
        prefix |= static_cast<uint32_t>(found[0]) << shift;
        left = found[1];
        if (round == 2) {
            equal_here = mine[found[0]];
            equal_before = __reduce_add_sync(0xffffffffu, lane < static_cast<int>(rank) ? ld_peer(&mine[found[0]], lane) : 0);
        }
    }
    // Rows with a larger key stay, and the first `left` of those with this one.  A warp has a run of rows.
    const int run = (r1 - r0 + kThreads - 1) / kThreads * 32, first = min(r0 + warp * run, r1), end = min(first + run, r1);
    int total;
    if (equal_here > 1) {                                     // (of one it does not matter which warp has it)
        int equal = 0;
        for (int j0 = first; j0 < end; j0 += 32) equal += __popc(__ballot_sync(0xffffffffu, j0 + lane < end && key_at(j0 + lane) == prefix));
        equal_before += warps_before(equal, red, &total);
    }
    const auto kept_of = [&](int j0, int& seen) {             // which of 32 rows stay; `seen`: equals so far
        const bool there = j0 + lane < end;
        const uint32_t k = there ? key_at(j0 + lane) : 0u;
        const unsigned eq = __ballot_sync(0xffffffffu, there && k == prefix);
        unsigned stay = __ballot_sync(0xffffffffu, there && k > prefix);
        if (eq) {
            stay |= __ballot_sync(0xffffffffu, there && k == prefix && seen + __popc(eq & ((1u << lane) - 1u)) < left);
            seen += __popc(eq);
        }
        return stay;
    };
    // (kept for the second walk where the keys are kept too: the bins of the second round are read by nobody any more)
    uint32_t* const staying = reinterpret_cast<uint32_t*>(hist[1]);
    static_assert(kKeysInSmem / 32 <= kBins, "a bit for every key");
    // holes: rows below m that go; moved: rows from m on that stay.  There are as many of one as of the other.
    int holes = 0, moved = 0;
    for (int j0 = first, seen = equal_before; j0 < end; j0 += 32) {
        const unsigned stay = kept_of(j0, seen);
        if (fits && lane == 0) staying[(j0 - r0) / 32] = stay;
        const unsigned below = j0 >= m ? 0u : j0 + 32 <= m ? 0xffffffffu : (1u << (m - j0)) - 1u;
        const unsigned there = end - j0 >= 32 ? 0xffffffffu : (1u << (end - j0)) - 1u;
        holes += __popc(~stay & below & there);
        moved += __popc(stay & ~below);
    }
    int holes_here, n_moves;
    int hole_at = warps_before(holes, red, &holes_here), moved_at = warps_before(moved, red, &n_moves);
    if (n_ranks > 1) {
        if (t == 0) { slots[2] = holes_here; slots[3] = n_moves; }
        cluster_sync();
        const int2 x = lane < static_cast<int>(n_ranks) ? ld_peer2(&slots[2], lane) : make_int2(0, 0);
        n_moves = __reduce_add_sync(0xffffffffu, x.y);
        hole_at += __reduce_add_sync(0xffffffffu, lane < static_cast<int>(rank) ? x.x : 0);
        moved_at += __reduce_add_sync(0xffffffffu, lane < static_cast<int>(rank) ? x.y : 0);
    }
    int2* const moves = a.moves + s.move0;
    const bool copies = a.pos_out != a.pos || a.mass_out != a.mass || a.kept_idx;
    for (int j0 = first, seen = equal_before; j0 < end; j0 += 32) {
        const unsigned stay = fits ? staying[(j0 - r0) / 32] : kept_of(j0, seen);
        const int j = j0 + lane;
        const unsigned below = j0 >= m ? 0u : j0 + 32 <= m ? 0xffffffffu : (1u << (m - j0)) - 1u;
        const unsigned there = end - j0 >= 32 ? 0xffffffffu : (1u << (end - j0)) - 1u;
        const unsigned hole = ~stay & below & there, from = stay & ~below, bit = 1u << lane, lower = bit - 1u;
        if (hole & bit) moves[hole_at + __popc(hole & lower)].y = j;
        if (from & bit) moves[moved_at + __popc(from & lower)].x = j;
        if (copies && (stay & below & bit)) {
            if (a.pos_out != a.pos) a.pos_out[row + j] = a.pos[row + j];
            if (a.mass_out != a.mass) a.mass_out[row + j] = a.mass[row + j];
            if (a.kept_idx) a.kept_idx[row + j] = j;
        }
        hole_at += __popc(hole);
        moved_at += __popc(from);
    }
    // (the writes to `moves` are visible to the CTA, to the cluster; and nobody reads another's shared memory any more)
    if (n_ranks > 1) cluster_sync();
    else __syncthreads();
    for (int i = static_cast<int>(rank) * kThreads + t; i < n_moves; i += static_cast<int>(n_ranks) * kThreads) {
        const int2 mv = moves[i];
        a.pos_out[row + mv.y] = a.pos[row + mv.x];
        a.mass_out[row + mv.y] = a.mass[row + mv.x];
        if (a.kept_idx) a.kept_idx[row + mv.y] = mv.x;
    }
    if (t == 0 && rank == 0) {
        a.n_moves[seq] = n_moves;
        if (a.kv_len_out) a.kv_len_out[s.index] = m;
    }
    if (a.max_moves <= kMovesInSelect && rank == 0) {         // (then no other kernel moves rows)
        const int pieces = static_cast<int>((a.row_bytes + kPiece - 1) / kPiece);
        for (int u = warp; u < n_moves * pieces * 2; u += kWarps) {
            const int2 mv = moves[u / (2 * pieces)];
            const int64_t off = static_cast<int64_t>(u / 2 % pieces) * kPiece;
            char* const base = static_cast<char*>(u & 1 ? a.v : a.k) + row * a.row_bytes + off;
            move_piece(base + mv.y * a.row_bytes, base + mv.x * a.row_bytes, static_cast<int>(min(static_cast<int64_t>(kPiece), a.row_bytes - off)), lane);
        }
    }
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictArgs a)
{
    __shared__ int64_t before[kMaxBatch + 1];
    pdl_wait();
    if (threadIdx.x == 0) {
        int64_t sum = 0;
        for (int b = 0; b < a.n_seq; ++b) {
            before[b] = sum;
            sum += a.n_moves[b];
        }
        before[a.n_seq] = sum;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, pieces = static_cast<int>((a.row_bytes + kPiece - 1) / kPiece);
    const int64_t units = before[a.n_seq] * pieces * 2, step = static_cast<int64_t>(gridDim.x) * (kMoveThreads / 32);
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + (threadIdx.x >> 5); u < units; u += step) {
        const int64_t i = u / (2 * pieces);
        const int w = static_cast<int>(u - i * 2 * pieces);
        int b = 0;
        while (i >= before[b + 1]) ++b;
        const EvictSeq& s = a.s[b];
        const int2 mv = a.moves[s.move0 + i - before[b]];
        const int64_t off = static_cast<int64_t>(w >> 1) * kPiece;
        char* const base = static_cast<char*>(w & 1 ? a.v : a.k) + s.kv_row * a.row_bytes + off;
        move_piece(base + mv.y * a.row_bytes, base + mv.x * a.row_bytes, static_cast<int>(min(static_cast<int64_t>(kPiece), a.row_bytes - off)), lane);
    }
}

}  // namespace

cudaError_t launch_cache_evict(const EvictArgs& a, cudaStream_t stream)
{
    static KernelSetup setup;
    int longest = 0;
    int64_t most = 0;
    for (int b = 0; b < a.n_seq; ++b) {
        longest = std::max(longest, a.s[b].n_kv);
        most += std::min(a.s[b].budget, std::max(0, a.s[b].n_kv - a.s[b].budget));
    }
    int cluster = 1;
    while (cluster < kMaxCluster && longest > cluster * kRowsPerCta) cluster *= 2;
    const int per_cta = (longest / cluster + 1 + kThreads - 1) / kThreads * kThreads;
    const size_t smem = sizeof(uint32_t) * static_cast<size_t>(std::min(per_cta, kKeysInSmem));
    cudaError_t e = setup_kernel(setup, reinterpret_cast<const void*>(evict_select_kernel), smem, 0);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_seq * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, evict_select_kernel, a);
    if (e != cudaSuccess || a.max_moves <= kMovesInSelect) return e;
    cfg.numAttrs = 1;
    const int64_t units = most * 2 * ((a.row_bytes + kPiece - 1) / kPiece);
    cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>((units + kMoveThreads / 32 - 1) / (kMoveThreads / 32), 8 * sm_count_of_current_device())));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, evict_move_kernel, a);
}

}  // namespace mvla
