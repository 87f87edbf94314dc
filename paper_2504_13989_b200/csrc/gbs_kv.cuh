// The paged KV cache as the kernels see it (included once per translation unit): addresses inside the pool, the items of a call,
// and H_128 on the 8 lanes that share a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gbs_internal.h"

namespace {

constexpr int KV_ROW = 64;                       // bytes of a row's packed codes (128 coordinates, 4 bits)
constexpr float KV_NORM = 0.08838834764831845f;  // 1 / sqrt(128)

// kernels wait for the launch before them here, having touched no memory
__device__ __forceinline__ void kv_wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void kv_let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// tokens of a sequence, whatever the array holds
__device__ __forceinline__ int kv_length(const gbs_kv_view& c, int seq)
{
    return min(max(c.lengths[seq], 0), c.max_pages << c.page_log);
}
// sequence of an item, or -1
__device__ __forceinline__ int kv_sequence(const gbs_kv_view& c, const int* seqs, int item)
{
    const int s = seqs ? seqs[item] : item;
    return (unsigned)s < (unsigned)c.n_seqs ? s : -1;
}
// page of a sequence's token, or -1
__device__ __forceinline__ int kv_page(const gbs_kv_view& c, int seq, int pos)
{
    const int id = c.page_table[(long long)seq * c.max_pages + (pos >> c.page_log)];
    return (unsigned)id < (unsigned)c.n_pages ? id : -1;
}
__device__ __forceinline__ unsigned char* kv_block(const gbs_kv_view& c, int page, int head)
{
    return c.pages + (long long)page * c.page_bytes + (long long)head * c.block_bytes;
}

// The item that row t belongs to (n_items: none), asked by a whole warp: how many of cu[1 .. n] are <= t, in a search that divides
// by 33 a step.  A step is one load, so 1024 items take two of them.  Ends for any contents of cu.
__device__ __forceinline__ int kv_item_of(const int* cu, int n, int t)
{
    int lo = 0, hi = n;
    const int lane = threadIdx.x & 31;
    while (hi > lo) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
        const unsigned below = __ballot_sync(0xffffffffu, at <= hi && cu[at] <= t);
        lo += __popc(below) * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// H_128 of a row that 8 neighbouring lanes share: lane l of them holds coordinates 8 l .. 8 l + 7 (v[0 .. 7]) and 64 + 8 l ..
// (v[8 .. 15]), the order in which 16-byte loads of 16-bit rows and 4-byte loads of codes are coalesced.  Unnormalised.
__device__ __forceinline__ void kv_hadamard(float v[16], int l8)
{
#pragma unroll
    for (int h = 1; h < 16; h <<= 1)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if ((i & h) == 0) {
                const float a = v[i], b = v[i + h];
                v[i] = a + b;
                v[i + h] = a - b;
            }
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) {
        const float sign = (l8 & h) ? -1.f : 1.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(v[i], sign, __shfl_xor_sync(0xffffffffu, v[i], h));
    }
}

__device__ __forceinline__ void kv_unpack_bf16(uint4 w, float v[8])
{
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 kv_pack_bf16(const float v[8])
{
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const unsigned*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

}  // namespace
