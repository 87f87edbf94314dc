// How an attention call is spread over the GPU (both kernels): tiles of query rows, pieces of the cache, and the join.
//
// Rows of an item are numbered token-major, (token, query head of the KV head); a tile is `rows` of them of one KV head, a segment is a
// tile with the part of the cache that any of its rows sees, cut into units of `unit` tokens.  The segments, in the order (item, tile, KV
// head), make one line, which the blocks share evenly: block b takes places b q .. (b + 1) q - 1, whatever segments they
// belong to.  So a batch of very different lengths is balanced without the host knowing one of them.  A segment takes as many places as it has
// units and `pad` more at its front, for what a segment costs apart from its units.  A segment whose units lie in one block is
// finished there; of one that several blocks share each leaves its sums in its workspace, and the join adds them up.  A
// block has at most two such segments: its first (slot 0) and its last (slot 1).
// Where no sequence is long, segments are not divided at all (pad < 0): each takes one place, and there is nothing to join.
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

struct KvLine {
    int entries, tiles, tile_rows;
    int unit_log;
    int pad;               // places of a segment before its units; -1: segments are not divided
    int least;             // a block takes at least so many places
    gbs_kv_div by_tiles;
    __device__ __forceinline__ int places(int units) const { return pad < 0 ? units != 0 : units != 0 ? units + pad : 0; }
};

__device__ __forceinline__ KvEntry kv_entry(const gbs_kv_attn& A, const KvLine& L, int index)
{
    KvEntry e;
    const int item = L.by_tiles(index), tile = index - item * L.tiles;
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
    e.row0 = tile * L.tile_rows;
    e.rows = max(0, min(count, A.max_tokens)) * A.group;
    e.before = e.length = e.lo = e.hi = e.units = 0;
    if (e.row0 >= e.rows) return e;
    e.before = length - count;
    e.length = length;
    const int last = min(e.rows, e.row0 + L.tile_rows) - 1;
    e.hi = kv_row_hi(A, e, A.by_group(last));
    e.lo = kv_row_lo(A, e, A.by_group(e.row0));
    // a tile that sees nothing is one unit too: its rows become 0
    e.units = 1;
    if (e.hi > e.lo) e.units = ((e.hi - 1) >> L.unit_log) - (e.lo >> L.unit_log) + 1;
    return e;
}

// A segment in a block's line.
struct KvSeg {
    int index, head;       // entry, KV head
    int at;                // its first place; below 0 where the block before has it
    KvEntry e;
};

// What of a segment is a block's: units skip .. skip + n - 1 of it.
struct KvPiece {
    int skip, n;
    bool starts, ends;     // it has the segment's first unit, its last one
};
__device__ __forceinline__ KvPiece kv_piece(const KvLine& L, const KvSeg& s, int places)
{
    if (L.pad < 0) return KvPiece{0, s.e.units, true, true};
    const int first = s.at + L.pad, end = first + s.e.units;
    return KvPiece{max(0, -first), min(places, end) - max(first, 0), first >= 0, end <= places};
}
// whether the block has places behind this segment
__device__ __forceinline__ bool kv_more(const KvLine& L, const KvSeg& s, int places) { return s.at + L.places(s.e.units) < places; }

__device__ __forceinline__ void kv_next(const gbs_kv_attn& A, const KvLine& L, KvSeg& s)
{
    s.at += L.places(s.e.units);
    if (++s.head < A.c.heads) return;
    s.head = 0;
    do {
        if (++s.index >= L.entries) { s.e.units = 0x3fffffff; return; }     // behind the last: a block has no places there
        s.e = kv_entry(A, L, s.index);
    } while (s.e.units == 0);
}

// The block's share: how many places, and in S the segment of the first one.  All threads of the block call it; `sh` is shared memory for
// one number a warp.  Places are counted in 64 bits: sums over all entries and heads.
template <int THREADS>
__device__ __forceinline__ int kv_share(const gbs_kv_attn& A, const KvLine& L, KvSeg* found, long long* sh)
{
    constexpr int WARPS = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int per = (L.entries + THREADS - 1) / THREADS, e0 = min(tid * per, L.entries), e1 = min(e0 + per, L.entries);
    long long mine = 0;
    KvEntry e = {};
    for (int i = e0; i < e1; ++i) {
        e = kv_entry(A, L, i);
        mine += L.places(e.units);
    }
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
    if (from < total && here <= from && from < here + mine * A.c.heads) {
        int i = e0;
        for (;; ++i) {
            if (per > 1) e = kv_entry(A, L, i);
            const long long n = (long long)L.places(e.units) * A.c.heads;
            if (from < here + n) break;
            here += n;
        }
        const int n = L.places(e.units), head = (int)((from - here) / n);
        found->index = i;
        found->head = head;
        found->at = (int)(here + (long long)head * n - from);               // 0 or below
        found->e = e;
    }
    __syncthreads();
    return from >= total ? 0 : (int)min(quota, total - from);
}

// What a block leaves for the join about the segment whose first unit it has and that ends in another block; blocks = 0: no such segment.
struct KvJoin {
    int index, head, blocks;
    int pad;
};
// the blocks behind have as many places each, or their rest
__device__ __forceinline__ KvJoin kv_join(const KvLine& L, const KvSeg& s, int places)
{
    const int beyond = s.at + L.pad + s.e.units - places;
    return KvJoin{s.index, s.head, 1 + (beyond + places - 1) / places, 0};
}

}  // namespace
