// What the items of a group have in common (gbs_kv_shared_attention): how many of their first tokens lie in the same pages, found in the page tables
// themselves, so that a result never depends on what a caller believes to be shared.  The attention kernels then run twice: over the prefix of each group, all
// rows of its items as if they were one item's, and over the rest of each item, where a row's sums over the prefix are added at the end.
//
// The tables of 64 sequences of 100 000 tokens are 6400 to 400 000 entries, which one SM would wait for the longest part of the call; a cluster of eight
// blocks compares them, a warp a slice of an item's entries with the same slice of the group's first item, and its first block makes the list of tiles.
#include <cooperative_groups.h>

#include "gbs_kv_sched.cuh"

namespace {

constexpr int BLOCKS = 8, THREADS = 1024, WARPS = THREADS / 32;
constexpr int NO_PART = -1;                      // of an item that shares nothing because it has no tokens, or no sequence

struct GroupArgs {
    gbs_kv_attn a;
    const int* groups;                           // null: one group of all items
    int n_groups, slices, tile_rows, unit_log, n_entries;
    int* common;                                 // [n_items][slices]: pages in common with the group's first item, as far as the slice tells
    int* shared;                                 // [n_items]
    KvEntry* entries;                            // [n_entries]
};

struct Range {
    int from, to;
};
__device__ __forceinline__ Range items_of(const GroupArgs& P, int g)
{
    if (!P.groups) return Range{0, P.a.n_items};
    const int from = min(max(P.groups[g], 0), P.a.n_items);
    return Range{from, min(max(P.groups[g + 1], from), P.a.n_items)};
}
// pages that lie wholly before an item's own tokens; NO_PART
__device__ __forceinline__ int pages_before(const gbs_kv_attn& A, const KvItem& x)
{
    return x.seq < 0 || x.count <= 0 ? NO_PART : max(x.length - x.count, 0) >> A.c.page_log;
}

// Group of an item, or -1, asked by a whole warp.
__device__ __forceinline__ int group_of(const GroupArgs& P, int item)
{
    if (!P.groups) return 0;
    if (item < P.groups[0]) return -1;
    const int g = kv_item_of(P.groups, P.n_groups, item);
    return g < P.n_groups ? g : -1;
}

__global__ __cluster_dims__(BLOCKS, 1, 1) __launch_bounds__(THREADS) void k_kv_groups(const __grid_constant__ GroupArgs P)
{
    __shared__ int tiles[GBS_KV_MAX_ITEMS];      // of each group, then of those before it
    __shared__ int sums[WARPS];
    const gbs_kv_attn& A = P.a;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, rank = blockIdx.x;
    kv_wait_before();
    kv_let_next();
    for (int i = rank * THREADS + threadIdx.x; i < A.n_items; i += BLOCKS * THREADS) P.shared[i] = 0;

    // ---- an item's slice against its group's first item's ----
    for (int job = rank * WARPS + w; job < A.n_items * P.slices; job += BLOCKS * WARPS) {
        const int i = job / P.slices, slice = job - i * P.slices;
        const int g = group_of(P, i);
        int found = NO_PART;
        if (g >= 0) {
            const KvItem x = kv_item(A, i);
            const int most = pages_before(A, x);
            if (most != NO_PART) {
                int lead = items_of(P, g).from;
                KvItem y = kv_item(A, lead);
                int y_most = pages_before(A, y);
                while (y_most == NO_PART && lead < i) {      // ends at the item itself at the latest
                    y = kv_item(A, ++lead);
                    y_most = pages_before(A, y);
                }
                const int n = max(min(most, y_most), 0), per = (n + P.slices - 1) / P.slices, from = min(slice * per, n), to = min(from + per, n);
                const int *a = A.c.page_table + (long long)x.seq * A.c.max_pages, *b = A.c.page_table + (long long)y.seq * A.c.max_pages;
                found = n;
                for (int j0 = from; j0 < to; j0 += 128) {
                    int u[4], v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = j0 + 32 * k + lane;
                        u[k] = j < to ? a[j] : 0;
                        v[k] = j < to ? b[j] : 0;
                    }
                    int first = 0x7fffffff;
#pragma unroll
                    for (int k = 3; k >= 0; --k)
                        if (u[k] != v[k]) first = j0 + 32 * k + lane;
                    first = __reduce_min_sync(0xffffffffu, first);
                    if (first != 0x7fffffff) {
                        found = first;
                        break;
                    }
                }
            }
        }
        if (lane == 0) P.common[job] = found;
    }
    __threadfence();
    cooperative_groups::this_cluster().sync();
    if (rank != 0) return;

    // ---- a warp a group: what all of its items share, and its rows ----
    for (int g = w; g < P.n_groups; g += WARPS) {
        const Range r = items_of(P, g);
        int pages = 0x7fffffff, members = 0;
        for (int job = r.from * P.slices + lane; job < r.to * P.slices; job += 32) {
            const int c = __ldcg(&P.common[job]);
            if (c != NO_PART) pages = min(pages, c);
            members += c != NO_PART && job % P.slices == 0;
        }
        pages = __reduce_min_sync(0xffffffffu, pages);
        members = __reduce_add_sync(0xffffffffu, members);
        if (members < 2) pages = 0;              // nothing is read twice
        if (lane == 0) {
            const int first = r.from < r.to ? min(max(A.cu ? A.cu[r.from] : r.from, 0), (int)A.n_tokens) : 0;
            const int end = r.from < r.to ? min(max(A.cu ? A.cu[r.to] : r.to, first), (int)A.n_tokens) : 0;
            tiles[g] = pages == 0 ? 0 : ((end - first) * A.group + P.tile_rows - 1) / P.tile_rows;
        }
        for (int i = r.from + lane; i < r.to; i += 32)
            if (__ldcg(&P.common[i * P.slices]) != NO_PART) P.shared[i] = pages << A.c.page_log;
    }
    __syncthreads();

    // ---- the groups' places in the list ----
    const int per = (P.n_groups + THREADS - 1) / THREADS, g0 = min((int)threadIdx.x * per, P.n_groups), g1 = min(g0 + per, P.n_groups);
    int mine = 0;
    for (int g = g0; g < g1; ++g) mine += tiles[g];
    int sum = mine;
#pragma unroll
    for (int h = 1; h < 32; h <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, h);
        if (lane >= h) sum += o;
    }
    if (lane == 31) sums[w] = sum;
    __syncthreads();
    int below = 0, all = 0;
    for (int i = 0; i < WARPS; ++i) {
        if (i < w) below += sums[i];
        all += sums[i];
    }
    int at = below + sum - mine;
    for (int g = g0; g < g1; ++g) {
        const int n = tiles[g];
        tiles[g] = at;
        at += n;
    }
    __syncthreads();
    all = min(all, P.n_entries);
    for (int e = threadIdx.x; e < P.n_entries; e += THREADS) {
        KvEntry x = {};
        x.seq = -1;
        if (e < all) {
            int lo = 0, hi = P.n_groups - 1;     // the last group that starts at e or before
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (tiles[mid] <= e) lo = mid;
                else hi = mid - 1;
            }
            const Range r = items_of(P, lo);
            KvItem y = {};
            int shared = 0;
            for (int i = r.from; i < r.to && shared == 0; ++i) {
                y = kv_item(A, i);
                shared = P.shared[i];
            }
            const int first = min(max(A.cu ? A.cu[r.from] : r.from, 0), (int)A.n_tokens), end = min(max(A.cu ? A.cu[r.to] : r.to, first), (int)A.n_tokens);
            x.seq = y.seq;
            x.first = first;
            x.rows = (end - first) * A.group;
            x.row0 = (e - tiles[lo]) * P.tile_rows;
            x.length = x.hi = shared;
            x.units = ((shared - 1) >> P.unit_log) + 1;
            if (shared == 0 || x.seq < 0 || x.row0 >= x.rows) x.units = 0;      // groups that overlap, whose numbers disagree
        }
        P.entries[e] = x;
    }
}

// up to so many rows of a group on average its prefix is read in tiles of 8 rows, beyond in tiles of 256
constexpr int FEW_PREFIX_ROWS = 32;
bool few_prefix(const gbs_kv_attn& A, int n_groups) { return A.n_tokens * A.group <= (int64_t)FEW_PREFIX_ROWS * n_groups; }
bool few_own(const gbs_kv_attn& A) { return (int64_t)A.max_tokens * A.group <= GBS_KV_FEW_ROWS; }
int64_t round_up(int64_t x) { return (x + 15) & ~(int64_t)15; }

struct Layout {
    int64_t attn, prefix, entries, shared, common, bytes;      // where each part starts
    int n_entries, slices;
};
Layout layout_of(const gbs_plan* p, const gbs_kv_attn& A, int n_groups)
{
    Layout l;
    const bool few = few_prefix(A, n_groups);
    const int tile = few ? 8 : 256;
    l.n_entries = (int)((A.n_tokens * A.group + tile - 1) / tile) + n_groups;
    l.slices = A.n_items < BLOCKS * WARPS ? BLOCKS * WARPS / (A.n_items > 0 ? A.n_items : 1) : 1;
    l.attn = 0;
    int64_t at = 0;
    if (few || few_own(A)) at = gbs_kv_few_workspace(p);
    if (!few || !few_own(A)) at = at > gbs_tc_kvattn_workspace(p) ? at : gbs_tc_kvattn_workspace(p);
    l.prefix = round_up(at);
    l.entries = l.prefix + round_up(A.n_tokens * A.n_heads * GBS_KV_PREFIX_ROW * (int64_t)sizeof(float));
    l.shared = l.entries + round_up(l.n_entries * (int64_t)sizeof(KvEntry));
    l.common = l.shared + round_up(A.n_items * (int64_t)sizeof(int));
    l.bytes = l.common + round_up((int64_t)A.n_items * l.slices * sizeof(int));
    return l;
}

}  // namespace

int64_t gbs_kv_shared_workspace(const gbs_plan* p, const gbs_kv_attn& A, int n_groups) { return layout_of(p, A, n_groups).bytes; }

int gbs_kv_shared_launch(const gbs_plan* p, const gbs_kv_attn& A, const int* groups, int n_groups, void* workspace, cudaStream_t stream)
{
    const Layout l = layout_of(p, A, n_groups);
    unsigned char* w = static_cast<unsigned char*>(workspace);
    const bool few = few_prefix(A, n_groups);
    GroupArgs G = {};
    G.a = A;
    G.groups = groups;
    G.n_groups = n_groups;
    G.slices = l.slices;
    G.tile_rows = few ? 8 : 256;
    G.unit_log = few ? 5 : 7;
    G.n_entries = l.n_entries;
    G.common = reinterpret_cast<int*>(w + l.common);
    G.shared = reinterpret_cast<int*>(w + l.shared);
    G.entries = reinterpret_cast<KvEntry*>(w + l.entries);
    int rc = gbs_kv_launch(p, k_kv_groups, dim3(BLOCKS), THREADS, 0, stream, G);
    if (rc != 0) return rc;
    gbs_kv_attn X = A;
    X.shared = G.shared;
    X.prefix = reinterpret_cast<float*>(w + l.prefix);
    gbs_kv_attn Y = X;
    Y.entries = G.entries;                       // of the prefixes: every row sees all of its group's
    Y.n_entries = l.n_entries;
    Y.causal = 0;
    Y.max_len = A.c.max_pages << A.c.page_log;
    rc = few ? gbs_kv_few_launch(p, Y, w, stream) : gbs_tc_kvattn_launch(p, Y, w, stream);
    if (rc != 0) return rc;
    return few_own(A) ? gbs_kv_few_launch(p, X, w, stream) : gbs_tc_kvattn_launch(p, X, w, stream);
}
