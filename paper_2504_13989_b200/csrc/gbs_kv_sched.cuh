// How an attention call is spread over the GPU (both kernels): tiles of query rows, pieces of the cache, and the join.
//
// Rows of an item are numbered token-major, (token, query head of the KV head); a tile is `rows` of them of one KV head, a segment is a
// tile with the part of the cache that any of its rows sees, cut into units of `unit` tokens.  The segments, in the order (item, tile, KV
// head), make one line of units, which the blocks share evenly: block b takes units b q .. (b + 1) q - 1, whatever segments they
// belong to.  So a batch of very different lengths is balanced without the host knowing one of them.  A segment that lies in one block is
// finished there; of one that several blocks share each leaves its sums in its workspace, and the join adds them up.  A
// block has at most two such segments: its first (slot 0) and its last (slot 1).
#pragma once

#include "gbs_kv.cuh"

namespace {

// One (item, tile): where its rows and its part of the cache are.
struct KvEntry {
    int seq;               // -1: none
    int first, rows;       // first row of the call's tensors, rows of the item (token-major, of one KV head)
    int row0;              // the tile's first row
    int before;            // cached tokens before the item's first
    int length;            // end of what may be read
    int lo, hi;            // tokens that some row of the tile sees: [lo, hi)
    int units;             // 0: no such tile
};

// a row sees tokens [row_lo, row_hi)
__device__ __forceinline__ int kv_row_hi(const gbs_kv_attn& A, const KvEntry& e, int token)
{
    return A.causal ? min(e.before + token + 1, e.length) : e.length;
}
__device__ __forceinline__ int kv_row_lo(const gbs_kv_attn& A, const KvEntry& e, int token)
{
    return A.window > 0 ? max(0, e.before + token - A.window + 1) : 0;
}

__device__ __forceinline__ KvEntry kv_entry(const gbs_kv_attn& A, int index, int tiles, int tile_rows, int unit)
{
    KvEntry e;
    const int item = index / tiles, tile = index - item * tiles;
    e.first = item;
    e.seq = A.seqs ? A.seqs[item] : item;
    int count = 1;
    if (A.cu) {
        e.first = A.cu[item];
        count = A.cu[item + 1] - e.first;
    }
    if ((unsigned)e.seq >= (unsigned)A.c.n_seqs) e.seq = -1;
    const int length = e.seq < 0 ? 0 : kv_length(A.c, e.seq);
    // no item has more rows than the call, nor a row outside it, whatever cu holds
    if (e.first < 0 || e.first > (int)A.n_tokens) count = 0;
    else count = min(count, (int)A.n_tokens - e.first);
    e.row0 = tile * tile_rows;
    e.rows = max(0, min(count, A.max_tokens)) * A.group;
    e.before = e.length = e.lo = e.hi = e.units = 0;
    if (e.row0 >= e.rows) return e;
    e.before = length - count;
    e.length = min(length, A.max_len);
    const int last = min(e.rows, e.row0 + tile_rows) - 1;
    e.hi = kv_row_hi(A, e, last / A.group);
    e.lo = kv_row_lo(A, e, e.row0 / A.group);
    // a tile that sees nothing is one unit too: its rows become 0
    e.units = 1;
    if (e.hi > e.lo) e.units = (e.hi - 1) / unit - e.lo / unit + 1;
    return e;
}

// A segment in a block's line: units 0 .. end of the line are the block's.
struct KvSeg {
    int index, head;       // entry, KV head
    int at;                // where its first unit lies; below 0 where the block before has its start
    KvEntry e;
};

__device__ __forceinline__ void kv_next(const gbs_kv_attn& A, KvSeg& s, int entries, int tiles, int tile_rows, int unit)
{
    s.at += s.e.units;
    if (++s.head < A.c.heads) return;
    s.head = 0;
    do {
        if (++s.index >= entries) { s.e.units = 0x3fffffff; return; }       // behind the last: never reached by a block's units
        s.e = kv_entry(A, s.index, tiles, tile_rows, unit);
    } while (s.e.units == 0);
}

struct KvLine {
    int entries, tiles, tile_rows, unit;
    int least;             // a block takes at least so many units; 0: whole segments, one after another
};

// The block's share: how many units, and the segment of the first one.  All threads of the block call it; `sh` holds 3 + 3 * warps ints.
// Units are counted in 64 bits: sums over all entries and heads.
template <int THREADS>
__device__ __forceinline__ int kv_share(const gbs_kv_attn& A, const KvLine& L, KvSeg& s, long long* sh)
{
    constexpr int WARPS = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int per = (L.entries + THREADS - 1) / THREADS, e0 = min(tid * per, L.entries), e1 = min(e0 + per, L.entries);
    long long mine = 0;
    for (int i = e0; i < e1; ++i) mine += kv_entry(A, i, L.tiles, L.tile_rows, L.unit).units;
    long long sum = mine;
#pragma unroll
    for (int h = 1; h < 32; h <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, sum, h);
        if (lane >= h) sum += o;
    }
    if (lane == 31) sh[w] = sum;
    __syncthreads();
    long long below = 0, all = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        if (i < w) below += sh[i];
        all += sh[i];
    }
    const long long total = all * A.c.heads;
    long long quota = (total + gridDim.x - 1) / gridDim.x;
    if (quota < L.least) quota = L.least;
    const long long from = quota * blockIdx.x;
    long long here = (below + sum - mine) * A.c.heads;                      // where this thread's first entry lies
    int* found = reinterpret_cast<int*>(sh + WARPS);
    __syncthreads();
    if (from < total && here <= from && from < here + mine * A.c.heads) {
        int i = e0;
        long long n;
        for (;; ++i) {
            n = kv_entry(A, i, L.tiles, L.tile_rows, L.unit).units;
            if (from < here + n * A.c.heads) break;
            here += n * A.c.heads;
        }
        const int head = (int)((from - here) / n);
        found[0] = i;
        found[1] = head;
        found[2] = (int)(here + head * n - from);                           // 0 or below
    }
    __syncthreads();
    if (from >= total) return 0;
    s.index = found[0];
    s.head = found[1];
    s.at = found[2];
    s.e = kv_entry(A, s.index, L.tiles, L.tile_rows, L.unit);
    return (int)min(quota, total - from);
}

// What a block leaves for the join about the segment that starts in it and ends in another block; blocks = 0: no such segment.
struct KvJoin {
    int index, head, blocks;
    int pad;
};

}  // namespace
