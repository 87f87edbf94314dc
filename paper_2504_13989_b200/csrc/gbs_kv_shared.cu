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
constexpr int NONE_YET = 0x7fffffff;

struct GroupArgs {
    gbs_kv_attn a;
    const int* groups;                           // null: one group of all items
    int n_groups, slices, tile_rows, unit_log, n_entries;
    int* shared;                                 // [n_items]
    KvEntry* entries;                            // [n_entries]
};

// What the block keeps of the items and the groups, in shared memory: every number that the call needs from elsewhere is fetched once.
struct Tables {
    int *seq, *before, *first;                   // [n_items]: the sequence, pages that lie wholly before the item's own tokens (NO_PART), its first row
    int *bounds, *lead, *common, *tiles;         // [n_groups] (bounds: and the end): first item, first item that takes part, pages that all have in common, members and then tiles
};
__host__ __device__ constexpr size_t table_ints(int n_items, int n_groups) { return 3 * (size_t)n_items + 4 * (size_t)n_groups + 1; }
static_assert(table_ints(GBS_KV_MAX_ITEMS, GBS_KV_MAX_ITEMS) * 4 + 1024 <= 227 * 1024, "one block's shared memory");

__global__ __cluster_dims__(BLOCKS, 1, 1) __launch_bounds__(THREADS) void k_kv_groups(const __grid_constant__ GroupArgs P)
{
    extern __shared__ int sm[];
    __shared__ int sums[WARPS];
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, rank = blockIdx.x, n = A.n_items, ng = P.n_groups;
    const Tables T = {sm, sm + n, sm + 2 * n, sm + 3 * n, sm + 3 * n + ng + 1, sm + 3 * n + 2 * ng + 1, sm + 3 * n + 3 * ng + 1};
    kv_wait_before();
    kv_let_next();

    // ---- the items and the groups: the same in all blocks ----
    for (int g = tid; g <= ng; g += THREADS) {
        T.bounds[g] = P.groups ? min(max(P.groups[g], 0), n) : g == 0 ? 0 : n;
        if (g < ng) {
            T.lead[g] = T.common[g] = NONE_YET;
            T.tiles[g] = 0;
        }
    }
    for (int i = tid; i < n; i += THREADS) {
        const KvItem x = kv_item(A, i);
        T.seq[i] = x.seq;
        T.first[i] = min(max(x.first, 0), (int)A.n_tokens);
        T.before[i] = x.seq < 0 || x.count <= 0 ? NO_PART : max(x.length - x.count, 0) >> A.c.page_log;
    }
    __syncthreads();
    // the last group that starts at an item or before it, if that reaches as far; -1
    const auto group_of = [&](int i) {
        if (i < T.bounds[0]) return -1;
        int lo = 0, hi = ng - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (T.bounds[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        return i < T.bounds[lo + 1] ? lo : -1;
    };
    for (int i = tid; i < n; i += THREADS) {
        const int g = T.before[i] != NO_PART ? group_of(i) : -1;
        if (g < 0) continue;
        atomicMin(&T.lead[g], i);
        atomicAdd(&T.tiles[g], 1);
    }
    // nobody adds to what the first block has not cleared yet
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();

    // ---- an item's slice against its group's first item's, a warp each ----
    int* common = cluster.map_shared_rank(T.common, 0);
    for (int job = rank * WARPS + w; job < n * P.slices; job += BLOCKS * WARPS) {
        const int i = job / P.slices, slice = job - i * P.slices;
        if (T.before[i] == NO_PART) continue;
        const int g = group_of(i);
        if (g < 0 || T.lead[g] == i) continue;
        const int lead = T.lead[g], pages = min(T.before[i], T.before[lead]);
        const int per = (pages + P.slices - 1) / P.slices, from = min(slice * per, pages), to = min(from + per, pages);
        const int *a = A.c.page_table + (long long)T.seq[i] * A.c.max_pages, *b = A.c.page_table + (long long)T.seq[lead] * A.c.max_pages;
        int found = pages;
        for (int j0 = from; j0 < to; j0 += 128) {
            int u[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = j0 + 32 * k + lane;
                u[k] = j < to ? a[j] : 0;
                v[k] = j < to ? b[j] : 0;
            }
            int first = NONE_YET;
#pragma unroll
            for (int k = 3; k >= 0; --k)
                if (u[k] != v[k]) first = j0 + 32 * k + lane;
            first = __reduce_min_sync(0xffffffffu, first);
            if (first != NONE_YET) {
                found = first;
                break;
            }
        }
        if (lane == 0) atomicMin(&common[g], found);
    }
    cluster.sync();
    if (rank != 0) return;

    // ---- what each item shares; the tiles of each group, and their places in the list ----
    const int per = (ng + THREADS - 1) / THREADS, g0 = min(tid * per, ng), g1 = min(g0 + per, ng);
    int mine = 0;
    for (int g = g0; g < g1; ++g) {
        const int pages = T.tiles[g] < 2 || T.common[g] == NONE_YET ? 0 : T.common[g];               // alone, nothing is read twice
        T.common[g] = pages;
        const int end = T.bounds[g + 1] < n ? T.first[T.bounds[g + 1]] : A.cu ? min(max(A.cu[n], 0), (int)A.n_tokens) : (int)A.n_tokens;
        const int rows = pages == 0 ? 0 : max(end - T.first[T.bounds[g]], 0) * A.group;
        T.tiles[g] = (rows + P.tile_rows - 1) / P.tile_rows;
        mine += T.tiles[g];
    }
    int sum = mine;
#pragma unroll
    for (int h = 1; h < 32; h <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, h);
        if (lane >= h) sum += o;
    }
    if (lane == 31) sums[w] = sum;
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
        const int g = T.before[i] != NO_PART ? group_of(i) : -1;
        P.shared[i] = g < 0 ? 0 : min(T.common[g], T.before[i]) << A.c.page_log;
    }
    int below = lane < w ? sums[lane] : 0, all = sums[lane];
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        below += __shfl_xor_sync(0xffffffffu, below, h);
        all += __shfl_xor_sync(0xffffffffu, all, h);
    }
    int at = below + sum - mine;
    for (int g = g0; g < g1; ++g) {
        const int tiles = T.tiles[g];
        T.tiles[g] = at;
        at += tiles;
    }
    __syncthreads();
    all = min(all, P.n_entries);
    for (int e = tid; e < P.n_entries; e += THREADS) {
        KvEntry x = {};
        x.seq = -1;
        if (e < all) {
            int lo = 0, hi = ng - 1;             // the last group whose tiles begin at e or before
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (T.tiles[mid] <= e) lo = mid;
                else hi = mid - 1;
            }
            const int end = T.bounds[lo + 1] < n ? T.first[T.bounds[lo + 1]] : A.cu ? min(max(A.cu[n], 0), (int)A.n_tokens) : (int)A.n_tokens;
            const int lead = T.lead[lo], shared = T.common[lo] << A.c.page_log;
            x.first = T.first[T.bounds[lo]];
            x.row0 = (e - T.tiles[lo]) * P.tile_rows;
            x.rows = max(end - x.first, 0) * A.group;
            // groups whose numbers fall may name items twice: what does not fit together has no units
            if (shared > 0 && lead < n && x.row0 >= 0 && x.row0 < x.rows) {
                x.seq = T.seq[lead];
                x.length = x.hi = min(shared, T.before[lead] << A.c.page_log);
                x.units = ((x.hi - 1) >> P.unit_log) + 1;
            }
        }
        P.entries[e] = x;
    }
}

// up to so many rows of a group on average its prefix is read in tiles of 8 rows, beyond in tiles of 128 or 256
constexpr int FEW_PREFIX_ROWS = 32;
bool few_prefix(const gbs_kv_attn& A, int n_groups) { return A.n_tokens * A.group <= (int64_t)FEW_PREFIX_ROWS * n_groups; }
bool few_own(const gbs_kv_attn& A) { return (int64_t)A.max_tokens * A.group <= GBS_KV_FEW_ROWS; }
// Up to 128 rows of a group on average, a block of the kernel for many rows has one tile of 128; up to 256 as well where prefixes are no longer than the units that all blocks
// get through in the time that queries and sums take (8 a block), by the table's width: 256 rows of 8 KV heads behind 6000 tokens 24 us instead of 26 and their join 5.7 instead of 7.4;
// behind 100 000 tokens one tile takes 1.4 times as long as two.
bool one_tile(const gbs_plan* p, const gbs_kv_attn& A, int n_groups)
{
    const int64_t rows = A.n_tokens * A.group, units = ((int64_t)A.c.max_pages << A.c.page_log) / 128;
    return rows <= 128ll * n_groups || (rows <= 256ll * n_groups && units * A.c.heads * n_groups <= 8ll * p->sm_count);
}
// Whether reading the prefixes once is likely to take less time than gbs_kv_attention does.  What an SM needs for 128 tokens, in microseconds: 0.63 for a tile of 8 rows, 2.5 (2.1 in one tile) up to 128
// rows, 2.9 for 256.  The lengths are not known here; without max_prefix the table's width stands for a prefix's.  Finding the groups, two more launches and their joins cost
// 20 to 45 us.  us with and without sharing, and the gain by this rule: 64 sequences behind 6000 tokens 54 and 98, 102; 14 behind 51 000 69 and 89, 74; 12 x 4 tokens behind 100 000 306 and 1102,
// 1030; but 10 behind 66 000, 2 KV heads, 64 and 55, 30; 17 behind 63 000, one KV head, 64 and 48, 26; 8 prompts of 250 behind 12 000 301 and 286, 30; 40 in 7 groups behind 8000 60 and 44,
// 19; 4 behind 300 27 and 12, 0.  Between 45 and 74 neither side was seen to lose by much.
constexpr double LEAST_GAIN = 45;
bool shares(const gbs_plan* p, const gbs_kv_attn& A, int n_groups, int64_t max_prefix)
{
    if (A.n_items == 0) return false;
    const auto tiles = [](double rows, int tile) { return (double)(int64_t)((rows + tile - 1) / tile); };
    const double most = (double)A.max_tokens * A.group, rows = (double)A.n_tokens * A.group / A.n_items, all = (double)A.n_tokens * A.group / n_groups;
    const double apart = most <= GBS_KV_FEW_ROWS ? tiles(most, 8) * 0.63 : most <= 128 ? 2.5 : tiles(rows, 256) * 2.9;
    const double once = all <= FEW_PREFIX_ROWS ? tiles(all, 8) * 0.63 : all <= 128 ? 2.1 : tiles(all, 256) * 2.9;
    const double longest = max_prefix > 0 ? (double)max_prefix : (double)((int64_t)A.c.max_pages << A.c.page_log);
    return (A.n_items * apart - n_groups * once) * A.c.heads / p->sm_count * longest / 128 > LEAST_GAIN;
}
int64_t round_up(int64_t x) { return (x + 15) & ~(int64_t)15; }

struct Layout {
    int64_t attn, prefix, entries, shared, bytes;      // where each part starts
    int n_entries;
};
Layout layout_of(const gbs_plan* p, const gbs_kv_attn& A, int n_groups)
{
    Layout l;
    const bool few = few_prefix(A, n_groups);
    const int tile = few ? 8 : 128;
    l.n_entries = (int)((A.n_tokens * A.group + tile - 1) / tile) + n_groups;
    l.attn = 0;
    int64_t at = 0;
    if (few || few_own(A)) at = gbs_kv_few_workspace(p);
    if (!few || !few_own(A)) at = at > gbs_tc_kvattn_workspace(p) ? at : gbs_tc_kvattn_workspace(p);
    l.prefix = round_up(at);
    l.entries = l.prefix + round_up(A.n_tokens * A.n_heads * GBS_KV_PREFIX_ROW * (int64_t)sizeof(float));
    l.shared = l.entries + round_up(l.n_entries * (int64_t)sizeof(KvEntry));
    l.bytes = l.shared + round_up(A.n_items * (int64_t)sizeof(int));
    return l;
}

}  // namespace

int64_t gbs_kv_shared_workspace(const gbs_plan* p, const gbs_kv_attn& A, int n_groups, int max_prefix)
{
    if (shares(p, A, n_groups, max_prefix)) return layout_of(p, A, n_groups).bytes;
    return few_own(A) ? gbs_kv_few_workspace(p) : gbs_tc_kvattn_workspace(p);
}

int gbs_kv_shared_launch(const gbs_plan* p, const gbs_kv_attn& A, const int* groups, int n_groups, int max_prefix, void* workspace, cudaStream_t stream)
{
    if (!shares(p, A, n_groups, max_prefix)) {
        gbs_kv_attn W = A;                       // max_len of an own part becomes one of a sequence
        W.fine = 1;                              // results are as precise whichever way they are found
        const int64_t width = (int64_t)A.c.max_pages << A.c.page_log;
        W.max_len = max_prefix > 0 && (int64_t)A.max_len + max_prefix < width ? A.max_len + max_prefix : (int)width;
        return few_own(A) ? gbs_kv_few_launch(p, W, workspace, stream) : gbs_tc_kvattn_launch(p, W, workspace, stream);
    }
    const Layout l = layout_of(p, A, n_groups);
    unsigned char* w = static_cast<unsigned char*>(workspace);
    const bool few = few_prefix(A, n_groups);
    GroupArgs G = {};
    G.a = A;
    G.groups = groups;
    G.n_groups = n_groups;
    G.slices = A.n_items < BLOCKS * WARPS ? BLOCKS * WARPS / A.n_items : 1;
    G.tile_rows = few ? 8 : one_tile(p, A, n_groups) ? 128 : 256;
    G.unit_log = few ? 5 : 7;
    G.n_entries = l.n_entries;
    G.shared = reinterpret_cast<int*>(w + l.shared);
    G.entries = reinterpret_cast<KvEntry*>(w + l.entries);
    const size_t smem = table_ints(A.n_items, n_groups) * sizeof(int);
    if (smem > 47 * 1024) {
        // the limit is the function's, for all threads of the process: always the same one, since a smaller call's may come between another's and its launch
        const cudaError_t e = cudaFuncSetAttribute((const void*)k_kv_groups, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)(table_ints(GBS_KV_MAX_ITEMS, GBS_KV_MAX_ITEMS) * sizeof(int)));
        if (e != cudaSuccess) return (int)e;
    }
    int rc = gbs_kv_launch(p, k_kv_groups, dim3(BLOCKS), THREADS, smem, stream, G);
    if (rc != 0) return rc;
    gbs_kv_attn X = A;
    X.shared = G.shared;
    X.prefix = reinterpret_cast<float*>(w + l.prefix);
    X.one_tile = (int64_t)A.max_tokens * A.group <= 128;
    gbs_kv_attn Y = X;
    Y.entries = G.entries;                       // of the prefixes: every row sees all of its group's
    Y.n_entries = l.n_entries;
    Y.one_tile = one_tile(p, A, n_groups);
    Y.causal = 0;
    Y.max_len = A.c.max_pages << A.c.page_log;
    rc = few ? gbs_kv_few_launch(p, Y, w, stream) : gbs_tc_kvattn_launch(p, Y, w, stream);
    if (rc != 0) return rc;
    return few_own(A) ? gbs_kv_few_launch(p, X, w, stream) : gbs_tc_kvattn_launch(p, X, w, stream);
}
