// Eviction from the paged KV cache (gbs_kv_evict): of a sequence longer than `keep` tokens each KV head keeps its first and last ones and, of those between, the ones with
// the largest mass.  Pages for what stays are taken first (gbs_kv_pages.cu), so that nothing is written over that is still to be read, whoever shares it; then
// a block (or a cluster of them) for each item and KV head finds what stays, all SMs move it, and last the tables change.
//
// What stays is found by digits from the highest down: a histogram of the first 11 bits of the weights, as integers of the same order, tells in which bin the last one
// that stays lies, then the next 11 bits of that bin's, then 10.  The threshold and how many that are equal to it stay give every token's
// place by prefix sums over positions: no sorting, and nothing depends on the order of threads.
#include <cooperative_groups.h>

#include "gbs_kv.cuh"

namespace {

constexpr int EACH = 8, HELD = 2;                // neighbouring tokens of a thread, and how many times so many it keeps in registers
constexpr int MOVE = 256, TOKENS = 2;            // threads of a block that moves, and tokens of one at a time
constexpr int BINS = 2048;

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

// A block, or a cluster of eight, per item and KV head.  A thread has EACH neighbouring tokens of every EACH * THREADS of its block's slice.  What it reads
// was written by launches that had ended before the one before it, which looks for pages, let it begin; only that one's status is waited for.
template <int THREADS, int BLOCKS>
__global__ __launch_bounds__(THREADS) void k_kv_select(const __grid_constant__ gbs_kv_eviction E)
{
    namespace cg = cooperative_groups;
    constexpr int PER = BINS / THREADS, WARPS = THREADS / 32;
    __shared__ int bins[BINS];
    __shared__ unsigned long long part[WARPS];
    __shared__ int found[2];                     // the bin, and how many of it stay
    __shared__ unsigned long long counts;        // of the slice: tokens that stay for sure, and those equal to the threshold
    const int tid = threadIdx.x, lane = tid & 31, rank = BLOCKS > 1 ? (int)cg::this_cluster().block_rank() : 0;
    const int row_of = blockIdx.x / BLOCKS, item = row_of / E.c.heads, head = row_of - item * E.c.heads;
    const auto all_blocks = [&] {
        if (BLOCKS > 1) cg::this_cluster().sync();
        else __syncthreads();
    };
    // of a block of the cluster
    const auto bins_of = [&](int r) { return BLOCKS > 1 ? cg::this_cluster().map_shared_rank(bins, r) : bins; };
    const auto counts_of = [&](int r) { return BLOCKS > 1 ? *cg::this_cluster().map_shared_rank(&counts, r) : counts; };

    const int seq = kv_sequence(E.c, E.seqs, item), length = seq < 0 ? 0 : kv_length(E.c, seq);
    const bool cut = length > E.keep;
    const long long row = ((long long)max(seq, 0) * E.c.heads + head) * E.width;
    const float* mass = E.mass + row;
    // the block's slice, and this thread's tokens of it that are kept in registers
    const int per = ((length + BLOCKS - 1) / BLOCKS + EACH - 1) / EACH * EACH, from = min(rank * per, length), to = min(from + per, length);
    const int lo = E.first, hi = length - E.recent;      // the tokens between
    const auto weight = [&](int pos) { return pos < to && pos < E.width ? mass[pos] : 0.f; };
    float w[HELD][EACH];
    if (cut)
#pragma unroll
        for (int x = 0; x < HELD; ++x)
#pragma unroll
            for (int k = 0; k < EACH; ++k) w[x][k] = weight(from + EACH * (THREADS * x + tid) + k);
    // f(first position of the thread's, its weights), by all threads of the block alike
    const auto each = [&](auto f) {
#pragma unroll
        for (int x = 0; x < HELD; ++x)
            if (from + EACH * THREADS * x < to) f(from + EACH * (THREADS * x + tid), w[x]);
        for (int p0 = from + HELD * EACH * THREADS; p0 < to; p0 += EACH * THREADS) {
            float v[EACH];
#pragma unroll
            for (int k = 0; k < EACH; ++k) v[k] = weight(p0 + EACH * tid + k);
            f(p0 + EACH * tid, v);
        }
    };
    unsigned threshold = 0;
    int want = E.keep - E.first - E.recent;
    const bool none = want == 0;
    if (cut && !none) {
        // ---- the threshold: `want` of the largest, digit by digit ----
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit < 2 ? 11 : 10, n = 1 << bits;
            for (int i = tid; i < BINS; i += THREADS) bins[i] = 0;
            __syncthreads();
            each([&](int pos, const float* v) {
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const unsigned u = order_of(v[k]);
                    const bool mine = pos + k >= lo && pos + k < hi && pos + k < to && (digit == 0 || (u >> (shift + bits)) == threshold);
                    const unsigned bin = mine ? (u >> shift) & (n - 1) : 0xffffffffu;
                    if (digit == 0) {            // the upper digits of most weights fall into few bins: those of a warp's that are alike are counted together
                        const unsigned same = __match_any_sync(0xffffffffu, bin);
                        if (mine && lane == __ffs(same) - 1) atomicAdd(&bins[bin], __popc(same));
                    } else if (mine) {
                        atomicAdd(&bins[bin], 1);
                    }
                }
            });
            all_blocks();
            // bins from the highest down, PER a thread
            int have[PER], sum = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int bin = n - 1 - PER * tid - k;
                have[k] = 0;
                if (bin >= 0)
#pragma unroll
                    for (int r = 0; r < BLOCKS; ++r) have[k] += bins_of(r)[bin];
                sum += have[k];
            }
            unsigned long long total;
            int above = (int)block_prefix<WARPS>((unsigned long long)sum, part, total);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (above < want && above + have[k] >= want) {
                    found[0] = n - 1 - PER * tid - k;
                    found[1] = want - above;
                }
                above += have[k];
            }
            all_blocks();                        // all have read the bins
            threshold = digit == 0 ? (unsigned)found[0] : threshold << bits | (unsigned)found[0];
            want = found[1];
        }
    }
    // above the threshold all stay, of those equal to it `want`, the lowest positions

    // ---- places ----
    const auto sort = [&](int pos, float x) -> int {     // 2: stays for sure, 1: equal to the threshold
        if (pos >= to) return 0;
        if (pos < lo || pos >= hi) return 2;
        const unsigned u = order_of(x);
        return none || u < threshold ? 0 : u > threshold ? 2 : 1;
    };
    unsigned long long before = 0;               // upper half: that stay for sure, lower: equal to the threshold
    if (cut && BLOCKS > 1) {                     // of the slices below
        unsigned long long mine = 0;
        each([&](int pos, const float* v) {
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int x = sort(pos + k, v[k]);
                mine += x == 2 ? 1ull << 32 : (unsigned long long)x;
            }
        });
        unsigned long long total;
        block_prefix<WARPS>(mine, part, total);
        if (tid == 0) counts = total;
        all_blocks();
        for (int r = 0; r < rank; ++r) before += counts_of(r);
        all_blocks();                            // a block stays until the others have read what it has
    }
    kv_wait_before();
    kv_let_next();
    if (E.status[item] != GBS_KV_DONE || !cut) { // nothing was done, or all of it stays
        const int stay = E.status[item] == GBS_KV_DONE ? length : 0;
        int* kept = E.kept + ((long long)item * E.c.heads + head) * E.keep;
        for (int j = THREADS * rank + tid; j < E.keep; j += THREADS * BLOCKS) kept[j] = j < stay ? j : -1;
        float* out = E.mass_out + row;
        if (out != mass)
            for (int j = THREADS * rank + tid; j < stay && j < E.width; j += THREADS * BLOCKS) out[j] = mass[j];
        return;
    }
    int* kept = E.kept + ((long long)item * E.c.heads + head) * E.keep;
    float* weights = E.weights + ((long long)item * E.c.heads + head) * E.keep;
    each([&](int pos, const float* v) {
        int how[EACH];
        unsigned long long mine = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            how[k] = sort(pos + k, v[k]);
            mine += how[k] == 2 ? 1ull << 32 : (unsigned long long)how[k];
        }
        unsigned long long total;
        const unsigned long long at = before + block_prefix<WARPS>(mine, part, total);
        int s = (int)(at >> 32), q = (int)(unsigned)at;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (how[k] == 2 || (how[k] == 1 && q < want)) {
                const int j = s + min(q, want);
                kept[j] = pos + k;
                weights[j] = v[k];
            }
            s += how[k] == 2;
            q += how[k] == 1;
        }
        before += total;
    });
}

// Rows of what stays: eight threads a token, 16 bytes of its codes each, two of them a scale as well, another one its weight.  The last block of an item lets its former pages go
// and enters the new ones into the table.
__global__ __launch_bounds__(MOVE, 5) void k_kv_evict_move(const __grid_constant__ gbs_kv_eviction E)
{
    __shared__ int last;
    kv_wait_before();
    kv_let_next();
    const int item = blockIdx.x / E.c.heads, head = blockIdx.x - item * E.c.heads, part = threadIdx.x & 7;
    const long long base = ((long long)item * E.c.heads + head) * E.keep;
    // a thread's part of TOKENS tokens, 32 apart; what does not depend on one another is asked for at once
    const int j0 = blockIdx.y * (TOKENS * MOVE / 8) + (threadIdx.x >> 3), step = gridDim.y * (TOKENS * MOVE / 8);
    int pos[TOKENS];
#pragma unroll
    for (int k = 0; k < TOKENS; ++k) pos[k] = j0 + 32 * k < E.keep ? E.kept[base + j0 + 32 * k] : -1;
    const int seq = kv_sequence(E.c, E.seqs, item);
    if (E.status[item] != GBS_KV_DONE) return;
    const int* fresh = E.fresh + (long long)item * E.keep_pages;
    int* table = E.c.page_table + (long long)seq * E.c.max_pages;
    const int length = kv_length(E.c, seq);
    float* out = E.mass_out + ((long long)seq * E.c.heads + head) * E.width;
    const int ps = 1 << E.c.page_log, scale_bytes = E.c.block_bytes / ps / 2 - KV_ROW;
    const int codes = (part >> 2) * ps * KV_ROW + 16 * (part & 3), scales = 2 * ps * KV_ROW + (part >> 2) * ps * scale_bytes;
    if (length <= E.keep) return;
    for (int j = j0; j < E.keep; j += step) {
        uint4 v[TOKENS];
        float2 sc[TOKENS];
        float weight[TOKENS];
        int page[TOKENS];
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
            const int from = pos[k] >= 0 ? table[pos[k] >> E.c.page_log] : -1;
            page[k] = pos[k] >= 0 ? fresh[(j + 32 * k) >> E.c.page_log] : 0;
            const bool ok = (unsigned)from < (unsigned)E.c.n_pages;
            const unsigned char* x = kv_block(E.c, ok ? from : 0, head);
            const int a = pos[k] & (ps - 1);
            v[k] = ok ? *reinterpret_cast<const uint4*>(x + codes + a * KV_ROW) : make_uint4(0, 0, 0, 0);
            sc[k] = make_float2(0.f, 0.f);
            if (ok && (part & 3) == 0) {
                if (scale_bytes == 8) sc[k] = *reinterpret_cast<const float2*>(x + scales + a * 8);
                else sc[k].x = *reinterpret_cast<const float*>(x + scales + a * 4);
            }
            weight[k] = part == 1 && pos[k] >= 0 ? E.weights[base + j + 32 * k] : 0.f;
        }
        int next[TOKENS];
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) next[k] = j + step + 32 * k < E.keep ? E.kept[base + j + step + 32 * k] : -1;
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
            if (pos[k] < 0) continue;
            const int to_j = j + 32 * k, b = to_j & (ps - 1);
            unsigned char* to = kv_block(E.c, page[k], head);
            *reinterpret_cast<uint4*>(to + codes + b * KV_ROW) = v[k];
            if ((part & 3) == 0) {
                if (scale_bytes == 8) *reinterpret_cast<float2*>(to + scales + b * 8) = sc[k];
                else *reinterpret_cast<float*>(to + scales + b * 4) = sc[k].x;
            }
            if (part == 1 && to_j < E.width) out[to_j] = weight[k];
        }
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) pos[k] = next[k];
    }
    __threadfence();
    __syncthreads();                             // the block has read the table and the length
    if (threadIdx.x == 0) last = atomicAdd(&E.arrived[item], 1) + 1 == E.c.heads * (int)gridDim.y;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int held = (int)(((unsigned)length + (1u << E.c.page_log) - 1) >> E.c.page_log);
    for (int j = threadIdx.x; j < held; j += MOVE) {
        const int page = table[j];
        if ((unsigned)page < (unsigned)E.c.n_pages) atomicSub(&E.c.refs[page], 1);
        if (j < E.keep_pages) table[j] = fresh[j];
    }
    if (threadIdx.x == 0) E.c.lengths[seq] = E.keep;
}

// Long sequences of few items and heads are looked through by clusters of 8 x 1024 threads, others by 256: 16 rows of 131 000 weights 168 us with a block of 1024 each.
constexpr int FEW = 256, MANY = 1024, CLUSTER = 8;

template <int THREADS, int BLOCKS>
int select(const gbs_plan* p, const gbs_kv_eviction& E, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)E.n_items * (unsigned)E.c.heads * BLOCKS);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = p->pdl ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = BLOCKS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return (int)cudaLaunchKernelEx(&cfg, k_kv_select<THREADS, BLOCKS>, E);
}

}  // namespace

int gbs_kv_evict_launch(const gbs_plan* p, const gbs_kv_eviction& E, cudaStream_t stream)
{
    int rc = gbs_kv_evict_pages_launch(p, E.c, E.seqs, E.n_items, E.keep, E.keep_pages, E.fresh, E.arrived, E.status, stream);
    const int64_t rows = (int64_t)E.n_items * E.c.heads, longest = (int64_t)E.c.max_pages << E.c.page_log;
    if (rc == 0) rc = longest > 2 * EACH * HELD * FEW && rows <= p->sm_count ? select<MANY, CLUSTER>(p, E, stream) : select<FEW, 1>(p, E, stream);
    // a block moves 64 tokens at a time; so many blocks of an item and KV head that all of them fill the GPU some times over
    const int64_t at_once = TOKENS * MOVE / 8, most = ((int64_t)E.keep + at_once - 1) / at_once, y = (int64_t)p->sm_count * 32 / rows + 1;
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_evict_move, dim3((unsigned)rows, (unsigned)(y < most ? y : most)), MOVE, 0, stream, E);
    return rc;
}
