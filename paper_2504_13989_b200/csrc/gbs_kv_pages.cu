// Bookkeeping of the paged KV cache (gbs_kv_extend, gbs_kv_fork, gbs_kv_free, gbs_kv_compact).
//
// refs[] is the whole truth about the pool: a page is free when its count is 0, and free pages are taken lowest first.  So the
// outcome of a call does not depend on the order in which threads run, and nothing has to be kept next to it.  Who gets which page
// follows from two prefix sums (pages wanted by the items before, free pages below), which one block computes: the items are at most
// a few thousand and the counters of a pool that fills the GPU a few megabytes.  What is large, the pages' contents and the tables'
// rows, is left to a second launch over all SMs.
#include "gbs_kv_alloc.cuh"

namespace {

constexpr int ONE = 1024;                        // threads of the one block that allocates
constexpr int COPY = 256;                        // threads of a block that copies pages
constexpr int PART = 128;                        // threads of a block that copies part of a page, or ends a sequence
constexpr int EACH = 4;                          // counters of a thread of the one block at a time

template <int WHAT>
__global__ __launch_bounds__(ONE) void k_kv_allocate(const __grid_constant__ AllocArgs A)
{
    extern __shared__ __align__(8) int sm[];
    __shared__ int part[32];
    kv_allocate_begin<ONE>(A.mask, sm);
    kv_wait_before();
    kv_let_next();
    kv_allocate<WHAT, ONE>(A, sm, part);
}

__device__ __forceinline__ void copy_words(unsigned char* to, const unsigned char* from, int bytes)
{
    for (int i = 4 * threadIdx.x; i < bytes; i += 4 * PART)
        *reinterpret_cast<unsigned*>(to + i) = *reinterpret_cast<const unsigned*>(from + i);
}
__device__ __forceinline__ void copy_16(unsigned char* to, const unsigned char* from, int bytes)
{
    for (int i = 16 * threadIdx.x; i < bytes; i += 16 * PART)
        *reinterpret_cast<uint4*>(to + i) = *reinterpret_cast<const uint4*>(from + i);
}

// One block per pair and KV head: its part of the last page's tokens; head 0 also shares the full pages.  The target's length is the
// one that the source had before the call.
__global__ __launch_bounds__(PART) void k_kv_share(const __grid_constant__ AllocArgs A)
{
    kv_wait_before();
    kv_let_next();
    const int i = blockIdx.x, head = blockIdx.y;
    if (A.status[i] != GBS_KV_DONE) return;
    const int dst = kv_sequence(A.c, A.seqs, i), src = kv_sequence(A.c, A.other, i);
    const int length = kv_length(A.c, dst), full = length >> A.c.page_log, ps = 1 << A.c.page_log, tail = length & (ps - 1);
    if (length == 0) return;
    if (head == 0) {
        const int* from = A.c.page_table + (long long)src * A.c.max_pages;
        int* to = A.c.page_table + (long long)dst * A.c.max_pages;
        for (int j = threadIdx.x; j < full; j += PART) {
            const int page = from[j];
            to[j] = page;
            if ((unsigned)page < (unsigned)A.c.n_pages) atomicAdd(&A.c.refs[page], 1);
        }
    }
    if (tail == 0) return;
    const int a = kv_page(A.c, src, length), b = kv_page(A.c, dst, length);
    if (a < 0 || b < 0) return;
    const unsigned char* from = kv_block(A.c, a, head);
    unsigned char* to = kv_block(A.c, b, head);
    const int scale_bytes = A.c.block_bytes / ps - 2 * KV_ROW;                   // both scales of a token
    copy_16(to, from, tail * KV_ROW);
    copy_16(to + ps * KV_ROW, from + ps * KV_ROW, tail * KV_ROW);
    to += 2 * ps * KV_ROW;
    from += 2 * ps * KV_ROW;
    copy_words(to, from, tail * scale_bytes / 2);
    copy_words(to + ps * scale_bytes / 2, from + ps * scale_bytes / 2, tail * scale_bytes / 2);
}

// One block per item; the exchange lets one of two blocks that name a sequence end it.
__global__ __launch_bounds__(PART) void k_kv_free(const __grid_constant__ AllocArgs A)
{
    __shared__ int length;
    kv_wait_before();
    kv_let_next();
    const int seq = kv_sequence(A.c, A.seqs, blockIdx.x);
    if (seq < 0) return;
    if (threadIdx.x == 0) length = min(max(atomicExch(&A.c.lengths[seq], 0), 0), A.c.max_pages << A.c.page_log);
    __syncthreads();
    const int held = (int)(((unsigned)length + (1u << A.c.page_log) - 1) >> A.c.page_log);
    const int* row = A.c.page_table + (long long)seq * A.c.max_pages;
    for (int j = threadIdx.x; j < held; j += PART) {
        const int page = row[j];
        if ((unsigned)page < (unsigned)A.c.n_pages) atomicSub(&A.c.refs[page], 1);
    }
}

struct CompactArgs {
    gbs_kv_view c, into;
    int *map, *n_live;
};

// new numbers of the pages in use
__global__ __launch_bounds__(ONE) void k_kv_number(const __grid_constant__ CompactArgs A)
{
    __shared__ int part[32];
    kv_wait_before();
    kv_let_next();
    Counters<EACH> now;
    now.load(A.c, EACH * threadIdx.x, 0);
    int live = 0;
    for (int p0 = 0; p0 < A.c.n_pages; p0 += EACH * ONE) {
        const int p = p0 + EACH * (int)threadIdx.x;
        int refs[EACH], used = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            refs[k] = now.r[k];
            used += refs[k] > 0;
        }
        now.load(A.c, p + EACH * ONE, 0);
        int total, r = live + block_prefix<ONE / 32>(used, part, total);
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (p + k < A.c.n_pages) {
                const bool moved = refs[k] > 0 && r < A.into.n_pages;
                A.map[p + k] = moved ? r : -1;
                if (moved) A.into.refs[r] = refs[k];
                r += refs[k] > 0;
            }
        live += total;
    }
    for (int p = live + threadIdx.x; p < A.into.n_pages; p += ONE) A.into.refs[p] = 0;
    if (threadIdx.x == 0) *A.n_live = live;
}

__global__ __launch_bounds__(COPY) void k_kv_move(const __grid_constant__ CompactArgs A)
{
    kv_wait_before();
    kv_let_next();
    const int ps = 1 << A.c.page_log;
    const long long entries = (long long)A.c.n_seqs * A.c.max_pages;
    for (long long e = (long long)blockIdx.x * COPY + threadIdx.x; e < entries; e += (long long)gridDim.x * COPY) {
        const int seq = (int)(e / A.c.max_pages), j = (int)(e - (long long)seq * A.c.max_pages);
        const int page = j < (int)(((unsigned)kv_length(A.c, seq) + ps - 1) >> A.c.page_log) ? A.c.page_table[e] : -1;
        A.into.page_table[e] = (unsigned)page < (unsigned)A.c.n_pages ? A.map[page] : -1;
    }
    for (int s = blockIdx.x * COPY + threadIdx.x; s < A.c.n_seqs; s += gridDim.x * COPY) A.into.lengths[s] = A.c.lengths[s];
    // pages one after another, eight pieces of a thread on their way at once; the next page's number is asked for ahead
    const int pieces = (int)(A.c.page_bytes / 16);
    int p = blockIdx.x, to = p < A.c.n_pages ? A.map[p] : -1;
    while (p < A.c.n_pages) {
        const int next = p + gridDim.x, next_to = next < A.c.n_pages ? A.map[next] : -1;
        if (to >= 0) {
            const uint4* from = reinterpret_cast<const uint4*>(A.c.pages + (long long)p * A.c.page_bytes);
            uint4* at = reinterpret_cast<uint4*>(A.into.pages + (long long)to * A.c.page_bytes);
            for (int i = threadIdx.x; i < pieces; i += 8 * COPY) {
                uint4 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i + k * COPY < pieces) v[k] = __ldcs(from + i + k * COPY);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i + k * COPY < pieces) __stcs(at + i + k * COPY, v[k]);
            }
        }
        p = next;
        to = next_to;
    }
}

template <int WHAT>
int allocate(const gbs_plan* p, const AllocArgs& A0, cudaStream_t stream)
{
    AllocArgs A = A0;
    A.mask = table_mask((unsigned)A.n_items);
    const size_t smem = table_bytes((unsigned)A.n_items);
    if (smem > 48 * 1024) {
        // the limit is the function's, for all threads of the process: always the same one, since a smaller call's may come between another's and its launch
        const cudaError_t e = cudaFuncSetAttribute((const void*)k_kv_allocate<WHAT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)table_bytes(GBS_KV_MAX_ITEMS));
        if (e != cudaSuccess) return (int)e;
    }
    return gbs_kv_launch(p, k_kv_allocate<WHAT>, dim3(1), ONE, smem, stream, A);
}

}  // namespace

int gbs_kv_extend_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, const int* counts, int n_items, int* status, cudaStream_t stream)
{
    return allocate<EXTEND>(p, {c, seqs, counts, n_items, status, 0}, stream);
}

int gbs_kv_fork_launch(const gbs_plan* p, const gbs_kv_view& c, const int* src, const int* dst, int n_items, int* status, cudaStream_t stream)
{
    const AllocArgs A = {c, dst, src, n_items, status, 0};
    const int e = allocate<FORK>(p, A, stream);
    if (e != 0) return e;
    return gbs_kv_launch(p, k_kv_share, dim3((unsigned)n_items, (unsigned)c.heads), PART, 0, stream, A);
}

int gbs_kv_free_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, int n_items, cudaStream_t stream)
{
    const AllocArgs A = {c, seqs, nullptr, n_items, nullptr, 0};
    return gbs_kv_launch(p, k_kv_free, dim3((unsigned)n_items), PART, 0, stream, A);
}

int gbs_kv_compact_launch(const gbs_plan* p, const gbs_kv_view& c, const gbs_kv_view& into, int* page_map, int* n_live, cudaStream_t stream)
{
    const CompactArgs A = {c, into, page_map, n_live};
    const int e = gbs_kv_launch(p, k_kv_number, dim3(1), ONE, 0, stream, A);
    if (e != 0) return e;
    return gbs_kv_launch(p, k_kv_move, dim3((unsigned)(p->sm_count * 8)), COPY, 0, stream, A);
}

int gbs_kv_evict_pages_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, int n_items, int keep, int keep_pages, int* fresh, int* arrived,
                              int* status, cudaStream_t stream)
{
    AllocArgs A = {c, seqs, nullptr, n_items, status, 0};
    A.keep = keep;
    A.keep_pages = keep_pages;
    A.fresh = fresh;
    A.arrived = arrived;
    return allocate<EVICT>(p, A, stream);
}
