// Bookkeeping of the paged KV cache (gbs_kv_extend, gbs_kv_fork, gbs_kv_free, gbs_kv_compact).
//
// refs[] is the whole truth about the pool: a page is free when its count is 0, and free pages are taken lowest first.  So the
// outcome of a call does not depend on the order in which threads run, and nothing has to be kept next to it.  Who gets which page
// follows from two prefix sums (pages wanted by the items before, free pages below), which one block computes: the items are at most
// a few thousand and the counters of a pool that fills the GPU a few megabytes.  What is large, the pages' contents and the tables'
// rows, is left to a second launch over all SMs.
#include "gbs_kv.cuh"

namespace {

constexpr int ONE = 1024;                        // threads of the one block that allocates
constexpr int COPY = 256;                        // threads of a block that copies pages
constexpr int PART = 128;                        // threads of a block that copies part of a page, or ends a sequence
constexpr int EACH = 4;                          // counters of a thread of the one block at a time (8 and 16: slower, 33 and 38 us for 30)

static_assert(ONE == 32 * 32, "a warp adds up what 32 warps have");
// Exclusive prefix sum over the block; `total` is the sum.  Two barriers; `part` holds 32 ints.
__device__ __forceinline__ int block_prefix(int v, int* part, int& total)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int h = 1; h < 32; h <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, s, h);
        if (lane >= h) s += o;
    }
    __syncthreads();                             // the last round's values have been read
    if (lane == 31) part[w] = s;
    __syncthreads();
    int below = lane < w ? part[lane] : 0, all = part[lane];
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        below += __shfl_xor_sync(0xffffffffu, below, h);
        all += __shfl_xor_sync(0xffffffffu, all, h);
    }
    total = all;
    return below + s - v;
}

// First item that names a sequence: a table in shared memory, keys and the lowest item of each.
struct FirstOf {
    int *key, *item;
    unsigned mask;
    __device__ __forceinline__ unsigned slot(int seq) const
    {
        unsigned h = ((unsigned)seq * 2654435761u) >> 7 & mask;
        for (;;) {                               // the table has room for twice the items
            const int was = atomicCAS(&key[h], -1, seq);
            if (was == -1 || was == seq) return h;
            h = (h + 1) & mask;
        }
    }
};

// EACH counters from p on; behind the last page: `behind`.  On their way while the ones before are worked on.
struct Counters {
    int r[EACH];
    __device__ __forceinline__ void load(const gbs_kv_view& c, int p, int behind)
    {
        if (p + EACH <= c.n_pages && (reinterpret_cast<uintptr_t>(c.refs) & 15) == 0) {
#pragma unroll
            for (int k = 0; k < EACH; k += 4) {
                const int4 v = *reinterpret_cast<const int4*>(c.refs + p + k);
                r[k] = v.x; r[k + 1] = v.y; r[k + 2] = v.z; r[k + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < EACH; ++k) r[k] = p + k < c.n_pages ? c.refs[p + k] : behind;
        }
    }
};

enum { EXTEND, FORK, EVICT };

struct AllocArgs {
    gbs_kv_view c;
    const int *seqs, *other;                     // extend: sequences and counts; fork: targets and sources
    int n_items;
    int* status;
    unsigned mask;
    // evict: tokens that a sequence keeps, their pages, and [n_items][keep_pages] numbers of pages for them
    int keep, keep_pages;
    int* fresh;
    int* arrived;                                // [n_items], becomes 0: what has been moved is counted there
};

// What an item asks for: its status, the tokens it will have, its first new page and how many.
struct Wish {
    int status, seq, length, first, need;
};
template <int WHAT>
__device__ __forceinline__ Wish wish_of(const AllocArgs& A, const FirstOf& f, int i)
{
    Wish w = {GBS_KV_BAD_INDEX, -1, 0, 0, 0};
    w.seq = kv_sequence(A.c, A.seqs, i);
    if (w.seq < 0) return w;
    if (f.item[f.slot(w.seq)] != i) {
        w.status = GBS_KV_DUPLICATE;
        return w;
    }
    const int ps = 1 << A.c.page_log, have = kv_length(A.c, w.seq);
    if (WHAT == FORK) {
        const int src = kv_sequence(A.c, A.other, i);
        if (src < 0) return w;
        if (have != 0) {
            w.status = GBS_KV_NOT_EMPTY;
            return w;
        }
        w.length = kv_length(A.c, src);
        w.first = w.length >> A.c.page_log;
        w.need = (w.length & (ps - 1)) != 0;
    } else if (WHAT == EVICT) {
        if (have > A.keep) w.need = A.keep_pages;
    } else {
        const int count = A.other ? A.other[i] : 1;
        if (count < 0) return w;
        if (count > (A.c.max_pages << A.c.page_log) - have) {
            w.status = GBS_KV_TOO_LONG;
            return w;
        }
        w.length = have + count;
        w.first = (int)(((unsigned)have + ps - 1) >> A.c.page_log);
        w.need = (int)(((unsigned)w.length + ps - 1) >> A.c.page_log) - w.first;
    }
    w.status = GBS_KV_DONE;
    return w;
}

// Shared memory: FirstOf's two arrays of mask + 1, then for each item where in the table page number 0 of the line of taken pages would be
// entered for it, and how many pages the items before it want (at the end, its new length).  Evict: the table is `fresh`, and lengths stay.
template <int WHAT>
__global__ __launch_bounds__(ONE) void k_kv_allocate(const __grid_constant__ AllocArgs A)
{
    extern __shared__ __align__(8) int sm[];
    __shared__ int part[32];
    int* const table = WHAT == EVICT ? A.fresh : A.c.page_table;
    const auto row_of = [&](const Wish& x, int i) { return WHAT == EVICT ? (long long)i * A.keep_pages : (long long)x.seq * A.c.max_pages + x.first; };
    FirstOf f = {sm, sm + A.mask + 1, A.mask};
    const int tid = threadIdx.x, n = A.n_items;
    long long* entry = reinterpret_cast<long long*>(sm + 2 * (A.mask + 1));
    int* before = reinterpret_cast<int*>(entry + n);
    for (unsigned i = tid; i <= A.mask; i += ONE) {
        f.key[i] = -1;
        f.item[i] = 0x7fffffff;
    }
    kv_wait_before();
    kv_let_next();
    Counters now;
    now.load(A.c, EACH * tid, 1);
    __syncthreads();
    for (int i = tid; i < n; i += ONE) {
        const int seq = kv_sequence(A.c, A.seqs, i);
        if (seq >= 0) atomicMin(&f.item[f.slot(seq)], i);
    }
    __syncthreads();
    // nothing that a wish goes by changes before the end, so a thread's first one is kept
    const Wish mine = wish_of<WHAT>(A, f, min(tid, n - 1));
    const auto wish = [&](int i) { return i == tid ? mine : wish_of<WHAT>(A, f, i); };

    // pages wanted before each item; more than the pool has need not be told apart
    int wanted = 0;
    for (int i0 = 0; i0 < n; i0 += ONE) {
        const int i = i0 + tid;
        const Wish w = i < n ? wish(i) : Wish{0, 0, 0, 0, 0};
        int total;
        const int at = wanted + block_prefix(min(w.need, 1 << 20), part, total);
        if (i < n) {
            before[i] = at;
            entry[i] = row_of(w, i) - at;
        }
        wanted = min(wanted + total, 0x3fffffff);
    }
    __syncthreads();

    // free pages, lowest first, go to the items in their order; what an item that is refused below has taken is given back there
    int found = 0;
    for (int p0 = 0; p0 < A.c.n_pages && found < wanted; p0 += EACH * ONE) {
        const int p = p0 + EACH * tid;
        unsigned free_bits = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) free_bits |= (now.r[k] == 0 ? 1u : 0u) << k;
        now.load(A.c, p + EACH * ONE, 1);
        int total, r = found + block_prefix(__popc(free_bits), part, total);
        if (free_bits && r < wanted) {
            int lo = 0, hi = n - 1;              // the last item with before[] <= r
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (before[mid] <= r) lo = mid;
                else hi = mid - 1;
            }
            for (; free_bits && r < wanted; free_bits &= free_bits - 1, ++r) {
                while (lo + 1 < n && before[lo + 1] <= r) ++lo;
                const int page = p + __ffs(free_bits) - 1;
                table[entry[lo] + r] = page;
                A.c.refs[page] = 1;
            }
        }
        found += total;
    }
    __syncthreads();

    // all wishes are read before a length changes: a fork's source may be another's target
    for (int i = tid; i < n; i += ONE) {
        Wish w = wish(i);
        if (w.status == GBS_KV_DONE && w.need > 0 && (long long)before[i] + w.need > found) {
            w.status = GBS_KV_NO_PAGES;
            for (int j = 0; j < w.need && before[i] + j < found; ++j)
                A.c.refs[table[row_of(w, i) + j]] = 0;
        }
        A.status[i] = w.status;
        if (WHAT == EVICT) A.arrived[i] = 0;
        before[i] = w.status == GBS_KV_DONE ? w.length : -1;
    }
    if (WHAT == EVICT) return;
    __syncthreads();
    for (int i = tid; i < n; i += ONE)
        if (before[i] >= 0) A.c.lengths[i == tid ? mine.seq : kv_sequence(A.c, A.seqs, i)] = before[i];
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
    Counters now;
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
        int total, r = live + block_prefix(used, part, total);
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

constexpr unsigned table_mask(unsigned n_items)
{
    unsigned mask = 63;
    while (mask + 1 < 2 * n_items) mask = 2 * mask + 1;
    return mask;
}
constexpr size_t table_bytes(unsigned n_items) { return (2 * ((size_t)table_mask(n_items) + 1) + 3 * (size_t)n_items) * sizeof(int); }
static_assert(table_bytes(GBS_KV_MAX_ITEMS) + 1024 <= 227 * 1024, "one block's shared memory");

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
