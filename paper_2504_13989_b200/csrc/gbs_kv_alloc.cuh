// Pages for the items of a call, found by one block (gbs_kv_extend, gbs_kv_fork, gbs_kv_evict).
//
// refs[] is the whole truth about the pool: a page is free when its count is 0, and free pages are taken lowest first.  So the outcome does not depend on the order in which threads run.  Who gets
// which page follows from two prefix sums (pages wanted by the items before, free pages below).
#pragma once

#include "gbs_kv.cuh"

namespace {

// Exclusive prefix sum over a block of WARPS warps; `total` is the sum.  Two barriers; `part` holds 32 ints.
template <int WARPS>
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
    int below = lane < w ? part[lane] : 0, all = lane < WARPS ? part[lane] : 0;
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

// Counters of a thread of the one block at a time (of 1024 threads; 8 and 16: slower, 33 and 38 us for 30): EACH from p on; behind the last page: `behind`.  On their way while the ones before are worked on.
template <int EACH>
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
// First, before anything is read:
template <int THREADS>
__device__ __forceinline__ void kv_allocate_begin(unsigned mask, int* sm)
{
    const FirstOf f = {sm, sm + mask + 1, mask};
    for (unsigned i = threadIdx.x; i <= mask; i += THREADS) {
        f.key[i] = -1;
        f.item[i] = 0x7fffffff;
    }
}
template <int WHAT, int THREADS>
__device__ __forceinline__ void kv_allocate(const AllocArgs& A, int* sm, int* part)
{
    constexpr int ONE = THREADS, EACH = THREADS == 1024 ? 4 : 8, WARPS = THREADS / 32;
    int* const table = WHAT == EVICT ? A.fresh : A.c.page_table;
    const auto row_of = [&](const Wish& x, int i) { return WHAT == EVICT ? (long long)i * A.keep_pages : (long long)x.seq * A.c.max_pages + x.first; };
    FirstOf f = {sm, sm + A.mask + 1, A.mask};
    const int tid = threadIdx.x, n = A.n_items;
    long long* entry = reinterpret_cast<long long*>(sm + 2 * (A.mask + 1));
    int* before = reinterpret_cast<int*>(entry + n);
    Counters<EACH> now;
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
        const int at = wanted + block_prefix<WARPS>(min(w.need, 1 << 20), part, total);
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
        int total, r = found + block_prefix<WARPS>(__popc(free_bits), part, total);
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

constexpr unsigned table_mask(unsigned n_items)
{
    unsigned mask = 63;
    while (mask + 1 < 2 * n_items) mask = 2 * mask + 1;
    return mask;
}
constexpr size_t table_bytes(unsigned n_items) { return (2 * ((size_t)table_mask(n_items) + 1) + 3 * (size_t)n_items) * sizeof(int); }
static_assert(table_bytes(GBS_KV_MAX_ITEMS) + 1024 <= 227 * 1024, "one block's shared memory");

}  // namespace
