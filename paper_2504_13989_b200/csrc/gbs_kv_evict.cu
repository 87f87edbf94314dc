// Eviction from the paged KV cache (gbs_kv_evict): of a sequence longer than `keep` tokens each KV head keeps its first and last ones and, of those between, the ones with
// the largest mass.  What stays moves into pages of its own, so that nothing is written over that is still to be read, whoever shares it: a block (or a cluster of them)
// for each item and KV head finds what stays, and one beside them the pages; then all SMs move it, and last the tables change.
//
// What stays is found by digits from the highest down: a histogram of the first 11 bits of the weights, as integers of the same order, tells in which bin the last one
// that stays lies, then the next 11 bits of that bin's, then 10.  The threshold and how many that are equal to it stay give every token's
// place by prefix sums over positions: no sorting, and nothing depends on the order of threads.
#include <cooperative_groups.h>

#include "gbs_kv_alloc.cuh"

namespace {

constexpr int EACH = 8, HELD = 2;                // neighbouring tokens of a thread, and how many times so many it keeps in registers
constexpr int MOVE = 256;                        // tokens that a block moves, and its threads
constexpr int BINS = 2048;
constexpr int FEW_ITEMS = 256;                   // up to so many, pages are looked for in the launch that looks for what stays
static_assert(table_bytes(FEW_ITEMS) <= BINS * sizeof(int), "in the same shared memory");

// weights as integers of the same order: NaN the largest, -0 as 0
__device__ __forceinline__ unsigned order_of(float x)
{
    if (x != x) return 0xffffffffu;
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Exclusive prefix sum over the block; `total` is the sum.
template <int WARPS>
__device__ __forceinline__ unsigned long long block_prefix(unsigned long long v, unsigned long long* part, unsigned long long& total)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    unsigned long long s = v;
#pragma unroll
    for (int h = 1; h < 32; h <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xffffffffu, s, h);
        if (lane >= h) s += o;
    }
    __syncthreads();                             // the last round's values have been read
    if (lane == 31) part[w] = s;
    __syncthreads();
    unsigned long long below = lane < w ? part[lane] : 0, all = lane < WARPS ? part[lane] : 0;
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        below += __shfl_xor_sync(0xffffffffu, below, h);
        all += __shfl_xor_sync(0xffffffffu, all, h);
    }
    total = all;
    return below + s - v;
}

// (a call of its own, so that the search for what stays keeps its registers)
template <int THREADS>
__device__ __noinline__ void find_pages(const gbs_kv_eviction& E, int* sm, int* part)
{
    kv_allocate<EVICT, THREADS>(AllocArgs{E.c, E.seqs, nullptr, E.n_items, E.status, E.mask, E.keep, E.keep_pages, E.fresh, E.arrived}, sm, part);
}

// A block, or a cluster of eight, per item and KV head.  A thread has EACH neighbouring tokens of every EACH * THREADS of its block's slice.  A sequence that one block can keep in registers is one
// block's in a cluster as well: how long sequences are is known here alone.  Neither what stays nor the pages for it need the other,
// so that one more block, the first one, looks for pages meanwhile; what this leaves of an item that is refused, the moving launch takes back.  (The two as launches of their own, each waiting for
// the one before, as with many items: 4 us more.)
template <int THREADS, int BLOCKS>
__global__ __launch_bounds__(THREADS, THREADS == 256 ? 6 : 1) void k_kv_select(const __grid_constant__ gbs_kv_eviction E)
{
    namespace cg = cooperative_groups;
    constexpr int PER = BINS / THREADS, WARPS = THREADS / 32;
    static_assert(HELD == 2 && EACH * THREADS < 1 << 16, "four counts in 64 bits");
    __shared__ __align__(8) int bins[BINS];      // (and what the search for pages needs)
    __shared__ int all[BLOCKS > 1 ? 2 : 1][BLOCKS > 1 ? BINS : 1];       // of the block; of the cluster, digit by digit in turn
    __shared__ unsigned long long part[WARPS];
    __shared__ int found[2];                     // the bin, and how many of it stay
    __shared__ int above_threshold, at_threshold;        // of the slice's tokens between
    __shared__ long long slices[BLOCKS];         // of each block: tokens that stay for sure (upper half), and that are equal to the threshold
    const int tid = threadIdx.x, lane = tid & 31, rank = BLOCKS > 1 ? (int)cg::this_cluster().block_rank() : 0;
    if (E.mask != 0 && blockIdx.x == 0) kv_allocate_begin<THREADS>(E.mask, bins);
    kv_wait_before();
    kv_let_next();
    if (E.mask != 0 && blockIdx.x < BLOCKS) {
        if (blockIdx.x == 0) find_pages<THREADS>(E, bins, reinterpret_cast<int*>(part));
        return;
    }
    const int row_of = blockIdx.x / BLOCKS - (E.mask != 0), item = row_of / E.c.heads, head = row_of - item * E.c.heads;
    const int seq = kv_sequence(E.c, E.seqs, item), length = seq < 0 ? 0 : kv_length(E.c, seq);
    const bool cut = length > E.keep;
    const int blocks = BLOCKS == 1 || length <= HELD * EACH * THREADS ? 1 : BLOCKS;
    if (cut && rank >= blocks) return;
    const auto all_blocks = [&] {
        if (BLOCKS > 1 && blocks > 1) cg::this_cluster().sync();
        else __syncthreads();
    };
    const long long row = ((long long)max(seq, 0) * E.c.heads + head) * E.width;
    const float* mass = E.mass + row;
    // the block's slice, and this thread's tokens of it that are kept in registers
    const int per = ((length + blocks - 1) / blocks + EACH - 1) / EACH * EACH, from = min(rank * per, length), to = min(from + per, length);
    const int lo = E.first, hi = length - E.recent;      // the tokens between
    const auto weight = [&](int pos) { return pos < to && pos < E.width ? mass[pos] : 0.f; };
    // a token between as a number above 0; 0: one that is not
    const auto key_of = [&](int pos, float x) { return pos >= lo && pos < hi && pos < to ? order_of(x) : 0u; };
    unsigned u[HELD][EACH];
    if (cut) {
        float w[HELD][EACH];
#pragma unroll
        for (int x = 0; x < HELD; ++x)
#pragma unroll
            for (int k = 0; k < EACH; ++k) w[x][k] = weight(from + EACH * (THREADS * x + tid) + k);
#pragma unroll
        for (int x = 0; x < HELD; ++x)
#pragma unroll
            for (int k = 0; k < EACH; ++k) u[x][k] = key_of(from + EACH * (THREADS * x + tid) + k, w[x][k]);
    }
    const int beyond = from + HELD * EACH * THREADS;     // tokens that are fetched again each time
    unsigned threshold = 0;
    int want = E.keep - E.first - E.recent;
    const bool none = want == 0;
    if (cut && !none) {
        if (blocks > 1)
            for (int i = tid; i < BINS; i += THREADS) all[0][i] = 0;
        if (tid == 0) above_threshold = 0;
        // ---- the threshold: `want` of the largest, digit by digit ----
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit < 2 ? 11 : 10, n = 1 << bits;
            for (int i = tid; i < BINS; i += THREADS) bins[i] = 0;
            if (blocks > 1 && digit == 0) all_blocks();          // nobody adds to what another block has not cleared yet
            else __syncthreads();
            const auto count = [&](unsigned v) {
                // (the upper digits of most weights fall into few bins; counting what is alike in a warp together first, by __match_any_sync: 37 us instead of 27 for 131 000
                // weights by eight blocks)
                if (digit == 0 ? v != 0 : v >> (shift + bits) == threshold) atomicAdd(&bins[(v >> shift) & (n - 1)], 1);
            };
#pragma unroll
            for (int x = 0; x < HELD; ++x)
                if (from + EACH * THREADS * x < to)
#pragma unroll
                    for (int k = 0; k < EACH; ++k) count(u[x][k]);
            for (int p0 = beyond; p0 < to; p0 += EACH * THREADS)
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const int pos = p0 + EACH * tid + k;
                    count(key_of(pos, weight(pos)));
                }
            __syncthreads();
            // bins from the highest down, PER a thread
            const int top = n - 1 - PER * tid;
            int mine[PER], have[PER], sum = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) have[k] = mine[k] = top - k >= 0 ? bins[top - k] : 0;
            if (BLOCKS > 1 && blocks > 1) {
                const int now = digit & 1;
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (mine[k] > 0)
#pragma unroll
                        for (int r = 0; r < BLOCKS; ++r) atomicAdd(&cg::this_cluster().map_shared_rank(all[now], r)[top - k], mine[k]);
                for (int i = tid; i < BINS; i += THREADS) all[now ^ 1][i] = 0;       // of the digit before: all have read it
                all_blocks();
#pragma unroll
                for (int k = 0; k < PER; ++k) have[k] = top - k >= 0 ? all[now][top - k] : 0;
            }
#pragma unroll
            for (int k = 0; k < PER; ++k) sum += have[k];
            unsigned long long total;
            int above = (int)block_prefix<WARPS>((unsigned long long)sum, part, total);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (above < want && above + have[k] >= want) {
                    found[0] = top - k;
                    found[1] = want - above;
                    at_threshold = mine[k];
                }
                above += have[k];
            }
            __syncthreads();
            if (blocks > 1) {                    // of the slice's, those above
                int over = 0;
#pragma unroll
                for (int k = 0; k < PER; ++k) over += top - k > found[0] ? mine[k] : 0;
                over = __reduce_add_sync(0xffffffffu, over);
                if (lane == 0 && over > 0) atomicAdd(&above_threshold, over);
            }
            threshold = digit == 0 ? (unsigned)found[0] : threshold << bits | (unsigned)found[0];
            want = found[1];
        }
    }
    // above the threshold all stay, of those equal to it `want`, the lowest positions

    // ---- places ----
    unsigned long long before = 0;               // upper half: tokens that stay for sure, lower: equal to the threshold
    if (BLOCKS > 1 && cut && blocks > 1) {       // of the slices below
        if (none) all_blocks();                  // nobody writes to a block that has not begun yet
        else __syncthreads();
        if (tid < BLOCKS) {
            const int ends = max(0, min(to, lo) - from) + max(0, to - max(from, hi));
            cg::this_cluster().map_shared_rank(slices, tid)[rank] = ((long long)(ends + (none ? 0 : above_threshold)) << 32) | (none ? 0 : at_threshold);
        }
        all_blocks();
        for (int r = 0; r < rank; ++r) before += (unsigned long long)slices[r];
    }
    int* kept = E.kept + ((long long)item * E.c.heads + head) * E.keep;
    if (!cut) {                                  // all of it stays
        for (long long j = THREADS * rank + tid; j < E.keep; j += THREADS * BLOCKS) kept[j] = j < length ? (int)j : -1;    // keep may be as large as an int
        float* out = E.mass_out + row;
        if (out != mass)                         // (of an item that is refused because an earlier one names its sequence, the same)
            for (int j = THREADS * rank + tid; j < length && j < E.width; j += THREADS * BLOCKS) out[j] = mass[j];
        return;
    }
    float* weights = E.weights + ((long long)item * E.c.heads + head) * E.keep;
    // which of a thread's EACH tokens stay for sure, and which are equal to the threshold
    const auto masks = [&](int pos, const unsigned* v, unsigned& sure, unsigned& equal) {
        sure = equal = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const bool end = pos + k < to && (pos + k < lo || pos + k >= hi);
            sure |= (unsigned)(end || (!none && v[k] > threshold)) << k;
            equal |= (unsigned)(!none && v[k] == threshold) << k;
        }
    };
    const auto write = [&](int pos, unsigned sure, unsigned equal, int s, int q) {
        if ((sure | equal) == 0) return;
        float w[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) w[k] = weight(pos + k);
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const bool is = sure >> k & 1, eq = equal >> k & 1;
            if (is || (eq && q < want)) {
                const int j = s + min(q, want);
                kept[j] = pos + k;
                weights[j] = w[k];
            }
            s += is;
            q += eq;
        }
    };
    unsigned sure[HELD], equal[HELD];
    unsigned long long mine = 0, total;
#pragma unroll
    for (int x = 0; x < HELD; ++x) {
        masks(from + EACH * (THREADS * x + tid), u[x], sure[x], equal[x]);
        mine |= (unsigned long long)__popc(sure[x]) << (32 * x + 16) | (unsigned long long)__popc(equal[x]) << (32 * x);
    }
    const unsigned long long at = block_prefix<WARPS>(mine, part, total);
    int s = (int)(before >> 32), q = (int)(unsigned)before;
#pragma unroll
    for (int x = 0; x < HELD; ++x) {
        write(from + EACH * (THREADS * x + tid), sure[x], equal[x], s + (int)(at >> (32 * x + 16) & 0xffff), q + (int)(at >> (32 * x) & 0xffff));
        s += (int)(total >> (32 * x + 16) & 0xffff);
        q += (int)(total >> (32 * x) & 0xffff);
    }
    for (int p0 = beyond; p0 < to; p0 += EACH * THREADS) {
        const int pos = p0 + EACH * tid;
        unsigned v[EACH], is, eq;
#pragma unroll
        for (int k = 0; k < EACH; ++k) v[k] = key_of(pos + k, weight(pos + k));
        masks(pos, v, is, eq);
        const unsigned long long here = block_prefix<WARPS>((unsigned long long)__popc(is) << 32 | (unsigned)__popc(eq), part, total);
        write(pos, is, eq, s + (int)(here >> 32), q + (int)(unsigned)here);
        s += (int)(total >> 32);
        q += (int)(unsigned)total;
    }
}

// Rows of what stays, MOVE tokens of a KV head a block: a thread finds where a token is and where it goes, and moves its scales and its weight; then eight threads a token move
// the codes, 16 bytes each.  The last block of an item lets its former pages go and enters the new ones into the table.  (Eight threads a token that find everything
// themselves: 313 instructions for four tokens, and 33 us instead of 20 for 290 000 tokens.)
__global__ __launch_bounds__(MOVE, 5) void k_kv_evict_move(const __grid_constant__ gbs_kv_eviction E)
{
    struct alignas(16) Way {
        const unsigned char* from;               // null: zeros
        unsigned char* to;                       // null: no such token
    };
    __shared__ Way ways[MOVE];
    __shared__ int last;
    kv_wait_before();
    kv_let_next();
    const int item = blockIdx.x / E.c.heads, head = blockIdx.x - item * E.c.heads;
    int j = blockIdx.y * MOVE + threadIdx.x;
    const long long base = ((long long)item * E.c.heads + head) * E.keep;
    int pos = j < E.keep ? E.kept[base + j] : -1;
    const int seq = kv_sequence(E.c, E.seqs, item);
    if (E.status[item] != GBS_KV_DONE) {         // nothing is done, and nothing stays (places that no sequence has are -1 already)
        const int most = min(E.keep, E.c.max_pages << E.c.page_log);
        for (; j < most; j += gridDim.y * MOVE) E.kept[base + j] = -1;
        return;
    }
    const int* fresh = E.fresh + (long long)item * E.keep_pages;
    int* table = E.c.page_table + (long long)seq * E.c.max_pages;
    const int length = kv_length(E.c, seq), ps = 1 << E.c.page_log;
    const bool asym = E.c.block_bytes > ps * (2 * KV_ROW + 8);
    if (length <= E.keep) return;
    for (long long first = blockIdx.y * MOVE; first < E.keep; first += gridDim.y * MOVE) {     // once, but for sequences of many millions
        Way way = {nullptr, nullptr};
        if (pos >= 0) {
            const int from = kv_page(E.c, seq, pos), a = pos & (ps - 1), b = j & (ps - 1);
            way.to = kv_block(E.c, fresh[j >> E.c.page_log], head);
            if (from >= 0) way.from = kv_block(E.c, from, head);
            if (asym) {
                const float2* x = reinterpret_cast<const float2*>(way.from + 2 * ps * KV_ROW) + a;
                const float2 k = from < 0 ? make_float2(0.f, 0.f) : x[0], v = from < 0 ? make_float2(0.f, 0.f) : x[ps];
                float2* y = reinterpret_cast<float2*>(way.to + 2 * ps * KV_ROW) + b;
                y[0] = k;
                y[ps] = v;
            } else {
                const float* x = reinterpret_cast<const float*>(way.from + 2 * ps * KV_ROW) + a;
                const float k = from < 0 ? 0.f : x[0], v = from < 0 ? 0.f : x[ps];
                float* y = reinterpret_cast<float*>(way.to + 2 * ps * KV_ROW) + b;
                y[0] = k;
                y[ps] = v;
            }
            if (j < E.width) E.mass_out[((long long)seq * E.c.heads + head) * E.width + j] = E.weights[base + j];
            if (from >= 0) way.from += a * KV_ROW;
            way.to += b * KV_ROW;
        }
        ways[threadIdx.x] = way;
        __syncthreads();
        const int part = threadIdx.x & 7, off = (part >> 2) * ps * KV_ROW + 16 * (part & 3);
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const unsigned char* from = ways[32 * k + (threadIdx.x >> 3)].from;
            v[k] = from ? *reinterpret_cast<const uint4*>(from + off) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (unsigned char* to = ways[32 * k + (threadIdx.x >> 3)].to) *reinterpret_cast<uint4*>(to + off) = v[k];
        if (gridDim.y * MOVE >= E.keep) break;
        j += gridDim.y * MOVE;               // keep is at most 2^27 where anything is cut: no overflow
        pos = j < E.keep ? E.kept[base + j] : -1;
        __syncthreads();                         // the ways have been read
    }
    __threadfence();
    __syncthreads();                             // the block has read the table and the length
    if (threadIdx.x == 0) last = atomicAdd(&E.arrived[item], 1) + 1 == E.c.heads * (int)gridDim.y;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int held = (int)(((unsigned)length + (1u << E.c.page_log) - 1) >> E.c.page_log);
    for (int i = threadIdx.x; i < held; i += MOVE) {
        const int page = table[i];
        if ((unsigned)page < (unsigned)E.c.n_pages) atomicSub(&E.c.refs[page], 1);
        if (i < E.keep_pages) table[i] = fresh[i];
    }
    if (threadIdx.x == 0) E.c.lengths[seq] = E.keep;
}

// Rows (items x KV heads) are looked through by 256 threads each, six rows an SM; by 1024, one an SM; or by clusters of eight blocks of 1024, of which some fifteen find eight SMs of one
// part of the GPU at a time.  The first keeps 4096 weights of a row in registers, the second 16 384; what is beyond is fetched four times.
// Which takes least goes by the tokens that a sequence can have, the table's width: lengths are not known here.  us of a call with a free and a fork before it (19), 512 of so many tokens stay:
//     rows      tokens 4000             9000             20 000            60 000            130 000      |  300 where 130 000 have room
//        8      27   27   27       39   31   31       62   40   31      160   79   35      319  141   45  |  23   27   27
//       16      27   28   29       41   33   34       63   41   45      161   80   53      320  142   67  |  25   27   27
//       48      27   29   39       41   33   47       64   43   74      164   82   86      324  144  116  |  25   27   37
//      144      30   33   64       43   39   81       68   49  161      174   92  192                     |  27   31   60
//      152      33   41   64       50   49   82       82   68  175      203  151  208                     |
//      296      36   49   98       57   62  131       93   83  308                                        |  29   43   90
//      768      78  112  232      125  140  308      202  197  771                                        |  41   80  193
// So where sequences are likely to be shorter than the table, the first is less of a loss than the others: they have to take a quarter less, and at most two rows an SM.
constexpr int FEW = 256, MANY = 1024, CLUSTER = 8;
enum Form { ROW_256, ROW_1024, ROW_CLUSTER };
Form form_of(const gbs_plan* p, int64_t rows, int64_t longest)
{
    const auto waves = [&](int64_t blocks) { return (double)((blocks + p->sm_count - 1) / p->sm_count); };
    const int64_t held = longest < HELD * EACH * FEW ? longest : HELD * EACH * FEW;
    const double few = (5.5 + 6e-4 * held + 2.3e-3 * (longest - held)) * (0.45 + 0.55 * waves(rows));
    const double many = waves(rows) * (4.5 + 9.2e-4 * longest), cluster = waves(10 * rows) * (12 + 1e-4 * longest);
    if (rows > 2 * p->sm_count || few <= 1.25 * (many < cluster ? many : cluster)) return ROW_256;
    return many <= cluster ? ROW_1024 : ROW_CLUSTER;
}

template <int THREADS, int BLOCKS>
int select(const gbs_plan* p, const gbs_kv_eviction& E, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(((unsigned)E.n_items * (unsigned)E.c.heads + (E.mask != 0)) * BLOCKS);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    // single blocks that began while the launch before still has most SMs would share the others: 32 us for 27 sequences of up to 7700 tokens behind a fork, 20 when they begin at its end
    attr[0].val.programmaticStreamSerializationAllowed = p->pdl && BLOCKS > 1 ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = BLOCKS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return (int)cudaLaunchKernelEx(&cfg, k_kv_select<THREADS, BLOCKS>, E);
}

}  // namespace

int gbs_kv_evict_launch(const gbs_plan* p, const gbs_kv_eviction& E0, cudaStream_t stream)
{
    gbs_kv_eviction E = E0;
    E.mask = E.n_items <= FEW_ITEMS ? table_mask((unsigned)E.n_items) : 0;
    int rc = E.mask != 0 ? 0 : gbs_kv_evict_pages_launch(p, E.c, E.seqs, E.n_items, E.keep, E.keep_pages, E.fresh, E.arrived, E.status, stream);
    const int64_t rows = (int64_t)E.n_items * E.c.heads, longest = (int64_t)E.c.max_pages << E.c.page_log;
    const Form form = form_of(p, rows, longest);
    if (rc == 0) rc = form == ROW_256 ? select<FEW, 1>(p, E, stream) : form == ROW_1024 ? select<MANY, 1>(p, E, stream) : select<MANY, CLUSTER>(p, E, stream);
    const int64_t most = E.keep < longest ? E.keep : longest, y = (most + MOVE - 1) / MOVE;
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_evict_move, dim3((unsigned)rows, (unsigned)(y < 65535 ? y : 65535)), MOVE, 0, stream, E);
    return rc;
}
