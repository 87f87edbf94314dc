// Eviction from the paged KV cache (gbs_kv_evict): of a sequence longer than `keep` tokens each KV head keeps its first and last ones and, of those between, the ones with
// the largest mass.  Pages for what stays are taken first (gbs_kv_pages.cu), so that nothing is written over that is still to be read, whoever shares it; then
// a block for each item and KV head finds what stays, all SMs move it, and last the tables change.
//
// What stays is found by digits from the highest down: a histogram of the first 11 bits of the weights, as integers of the same order, tells in which bin the last one
// that stays lies, then the next 11 bits of that bin's, then 10.  The threshold and how many that are equal to it stay give every token's
// place by prefix sums over positions: no sorting, and nothing depends on the order of threads.
#include "gbs_kv.cuh"

namespace {

constexpr int SELECT = 1024, EACH = 8;           // threads of a block that selects, and neighbouring tokens of one
constexpr int MOVE = 256;
constexpr int BINS = 2048;

// weights as integers of the same order: NaN the largest, -0 as 0
__device__ __forceinline__ unsigned order_of(float x)
{
    if (x != x) return 0xffffffffu;
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Exclusive prefix sum over the block; `total` is the sum.
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
    unsigned long long below = lane < w ? part[lane] : 0, all = part[lane];
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        below += __shfl_xor_sync(0xffffffffu, below, h);
        all += __shfl_xor_sync(0xffffffffu, all, h);
    }
    total = all;
    return below + s - v;
}

// One block per item and KV head.
__global__ __launch_bounds__(SELECT) void k_kv_select(const __grid_constant__ gbs_kv_eviction E)
{
    __shared__ int bins[BINS];
    __shared__ unsigned long long part[32];
    __shared__ int found[2];                     // the bin, and how many of it stay
    kv_wait_before();
    kv_let_next();
    const int item = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
    int* kept = E.kept + ((long long)item * E.c.heads + head) * E.keep;
    const bool done = E.status[item] == GBS_KV_DONE;
    const int seq = done ? kv_sequence(E.c, E.seqs, item) : -1, length = seq < 0 ? 0 : kv_length(E.c, seq);
    const long long row = ((long long)max(seq, 0) * E.c.heads + head) * E.width;
    const float* mass = E.mass + row;
    float* out = E.mass_out + row;
    if (length <= E.keep) {                      // all of it stays, or nothing was done
        for (int j = tid; j < E.keep; j += SELECT) kept[j] = j < length ? j : -1;
        if (out != mass)
            for (int j = tid; j < length && j < E.width; j += SELECT) out[j] = mass[j];
        return;
    }
    const int lo = E.first, hi = length - E.recent;      // the tokens between
    const auto weight = [&](int pos) { return pos < E.width ? mass[pos] : 0.f; };

    // ---- the threshold: `want` of the largest, digit by digit ----
    unsigned threshold = 0;
    int want = E.keep - E.first - E.recent;
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit < 2 ? 11 : 10, n = 1 << bits;
        for (int i = tid; i < BINS; i += SELECT) bins[i] = 0;
        __syncthreads();
        for (int pos = lo + tid; pos < hi; pos += SELECT) {
            const unsigned u = order_of(weight(pos));
            if (digit == 0 || (u >> (shift + bits)) == threshold) atomicAdd(&bins[(u >> shift) & (n - 1)], 1);
        }
        __syncthreads();
        // bins from the highest down, two a thread
        const int top = n - 1 - 2 * tid, a = top >= 0 ? bins[top] : 0, b = top >= 1 ? bins[top - 1] : 0;
        unsigned long long total;
        const int above = (int)block_prefix((unsigned long long)(a + b), part, total);
        if (above < want && above + a >= want) { found[0] = top; found[1] = want - above; }
        else if (above + a < want && above + a + b >= want) { found[0] = top - 1; found[1] = want - above - a; }
        __syncthreads();
        if (want > 0) {
            threshold = digit == 0 ? (unsigned)found[0] : threshold << bits | (unsigned)found[0];
            want = found[1];
        }
        __syncthreads();
    }
    // above the threshold all stay, of those equal to it `want`, the lowest positions; with nothing to take none is above
    const bool none = E.keep == E.first + E.recent;

    // ---- places ----
    long long before = 0, equal_before = 0;      // that stay for sure, and that are equal to the threshold
    for (int p0 = 0; p0 < length; p0 += SELECT * EACH) {
        const int pos = p0 + EACH * tid;
        float w[EACH];
        unsigned sure = 0, equal = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            w[k] = pos + k < length ? weight(pos + k) : 0.f;
            const bool between = pos + k >= lo && pos + k < hi;
            const unsigned u = order_of(w[k]);
            sure |= (unsigned)(pos + k < length && (!between || (!none && u > threshold))) << k;
            equal |= (unsigned)(between && !none && u == threshold) << k;
        }
        unsigned long long total;
        const unsigned long long at = block_prefix((unsigned long long)__popc(sure) << 32 | (unsigned)__popc(equal), part, total);
        long long s = before + (long long)(at >> 32), q = equal_before + (long long)(at & 0xffffffffu);
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const bool eq = equal >> k & 1;
            if ((sure >> k & 1) || (eq && q < want)) {
                const long long j = s + min(q, (long long)want);
                kept[j] = pos + k;
                if (j < E.width) out[j] = w[k];
            }
            s += sure >> k & 1;
            q += eq;
        }
        before += (long long)(total >> 32);
        equal_before += (long long)(total & 0xffffffffu);
    }
}

// Rows of what stays: eight threads a token, 16 bytes of its codes each, two of them a scale as well.
__global__ __launch_bounds__(MOVE) void k_kv_evict_move(const __grid_constant__ gbs_kv_eviction E)
{
    kv_wait_before();
    kv_let_next();
    const int item = blockIdx.x / E.c.heads, head = blockIdx.x - item * E.c.heads;
    if (E.status[item] != GBS_KV_DONE) return;
    const int seq = kv_sequence(E.c, E.seqs, item);
    if (kv_length(E.c, seq) <= E.keep) return;
    const int* kept = E.kept + ((long long)item * E.c.heads + head) * E.keep;
    const int* fresh = E.fresh + (long long)item * E.keep_pages;
    const int ps = 1 << E.c.page_log, scale_bytes = E.c.block_bytes / ps / 2 - KV_ROW, part = threadIdx.x & 7;
    for (int j = blockIdx.y * (MOVE / 8) + (threadIdx.x >> 3); j < E.keep; j += gridDim.y * (MOVE / 8)) {
        const int pos = kept[j], from = kv_page(E.c, seq, pos), a = pos & (ps - 1), b = j & (ps - 1);
        unsigned char* to = kv_block(E.c, fresh[j >> E.c.page_log], head);
        const unsigned char* x = kv_block(E.c, max(from, 0), head);
        const int codes = (part >> 2) * ps * KV_ROW + 16 * (part & 3);
        uint4 v = *reinterpret_cast<const uint4*>(x + codes + a * KV_ROW);
        if (from < 0) v = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(to + codes + b * KV_ROW) = v;
        if ((part & 3) == 0) {
            const int scales = 2 * ps * KV_ROW + (part >> 2) * ps * scale_bytes;
            for (int k = 0; k < scale_bytes; k += 4)
                *reinterpret_cast<float*>(to + scales + b * scale_bytes + k) = from < 0 ? 0.f : *reinterpret_cast<const float*>(x + scales + a * scale_bytes + k);
        }
    }
}

// One block per item: its former pages are let go, and the new ones enter the table.
__global__ __launch_bounds__(128) void k_kv_evict_end(const __grid_constant__ gbs_kv_eviction E)
{
    kv_wait_before();
    kv_let_next();
    const int item = blockIdx.x;
    if (E.status[item] != GBS_KV_DONE) return;
    const int seq = kv_sequence(E.c, E.seqs, item), length = kv_length(E.c, seq);
    if (length <= E.keep) return;
    __syncthreads();                             // all have read the length
    int* row = E.c.page_table + (long long)seq * E.c.max_pages;
    const int held = (int)(((unsigned)length + (1u << E.c.page_log) - 1) >> E.c.page_log);
    for (int j = threadIdx.x; j < held; j += 128) {
        const int page = row[j];
        if ((unsigned)page < (unsigned)E.c.n_pages) atomicSub(&E.c.refs[page], 1);
        if (j < E.keep_pages) row[j] = E.fresh[(long long)item * E.keep_pages + j];
    }
    if (threadIdx.x == 0) E.c.lengths[seq] = E.keep;
}

}  // namespace

int gbs_kv_evict_launch(const gbs_plan* p, const gbs_kv_eviction& E, cudaStream_t stream)
{
    int rc = gbs_kv_evict_pages_launch(p, E.c, E.seqs, E.n_items, E.keep, E.keep_pages, E.fresh, E.status, stream);
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_select, dim3((unsigned)E.n_items, (unsigned)E.c.heads), SELECT, 0, stream, E);
    // a block moves 32 tokens at a time; so many blocks of an item and KV head that all of them fill the GPU some times over
    const int64_t rows = (int64_t)E.n_items * E.c.heads, most = ((int64_t)E.keep + MOVE / 8 - 1) / (MOVE / 8);
    const int64_t x = (int64_t)p->sm_count * 32 / rows + 1;
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_evict_move, dim3((unsigned)rows, (unsigned)(x < most ? x : most)), MOVE, 0, stream, E);
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_evict_end, dim3((unsigned)E.n_items), 128, 0, stream, E);
    return rc;
}
