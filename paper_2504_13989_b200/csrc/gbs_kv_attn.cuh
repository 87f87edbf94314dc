// What the two attention kernels over the paged KV cache share: numbers out of codes, partial results and their join.
#pragma once

#include <cuda_fp16.h>

#include "gbs_kv_sched.cuh"

namespace {

constexpr float NONE = -1e30f;                       // maximum of no scores
constexpr float W_UP = 64.f;                         // weights are kept at 64 times their size relative to the largest

// floats of a partial result: sums of w c, then for each row m, the total, the sum of p mid, and M
template <int ROWS>
constexpr int KV_PART = ROWS * 128 + 4 * ROWS;

// totals of the kernel for many rows (tiles of 256) are 64 times their size
template <int ROWS>
constexpr float KV_TOTAL_LOG = ROWS == 256 ? 6.f : 0.f;

struct KvAttnArgs {
    gbs_kv_attn a;
    KvLine line;
    float* parts;                                    // [blocks][2][PART]
    KvJoin* joins;                                   // [blocks]
    int blocks;                                      // of the kernel whose sums are joined
    int* status;
};

// Whether a wait counts as one that ran out: in the self-test's instances, those with the given code in a block's segment of the given number.
template <bool TEST, typename Args>
__device__ __forceinline__ bool kv_lost(const Args& P, volatile int* abort_flag, int code, int segment)
{
    if (!TEST || code != P.a.lost_code || segment != P.a.lost_segment) return false;
    *abort_flag = 1;
    atomicCAS(P.status, 0, code);
    return true;
}

__device__ __forceinline__ unsigned as_u(__half2 x) { return *reinterpret_cast<unsigned*>(&x); }
__device__ __forceinline__ __half2 as_h(unsigned x) { return *reinterpret_cast<__half2*>(&x); }

__device__ __forceinline__ float kv_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// (x & mask) ^ with, one operation
__device__ __forceinline__ unsigned kv_and_xor(unsigned x, unsigned mask, unsigned with)
{
    unsigned y;
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(y) : "r"(x), "r"(mask), "r"(with));
    return y;
}
// Nibbles (i, i + 4) of a word, i = 0 .. 3, as pairs in fp16, -8 .. 7.  A symmetric code c is taken as c ^ 8 = c + 8 of four bits, an asymmetric one counts
// from the middle of its range, 8: sums of products with codes that are all positive would be large next to what is left of them once lo is added,
// and the matrix unit drops what lies below their last bit (130000 tokens in one block, a broad softmax: a tenth of the result, with codes from 0).
template <bool ASYM>
__device__ __forceinline__ void kv_codes_f16(unsigned w, unsigned out[4])
{
    constexpr unsigned LOW = ASYM ? 0x64006400u : 0x64086408u, HIGH = ASYM ? 0x64006400u : 0x64806480u;
    const __half2 off = __float2half2_rn(1032.f), off16 = __float2half2_rn(-72.f), by = __float2half2_rn(0.0625f);
    const unsigned w8 = w >> 8;
    out[0] = as_u(__hsub2(as_h(kv_and_xor(w, 0x000f000fu, LOW)), off));
    out[1] = as_u(__hfma2(as_h(kv_and_xor(w, 0x00f000f0u, HIGH)), by, off16));
    out[2] = as_u(__hsub2(as_h(kv_and_xor(w8, 0x000f000fu, LOW)), off));
    out[3] = as_u(__hfma2(as_h(kv_and_xor(w8, 0x00f000f0u, HIGH)), by, off16));
}

// sums of w c, of p and of p mid -> the result: sum / 64 2^(M - m) / total + extra / total, turned back
__device__ __forceinline__ void kv_finish(float y[16], int l8, float top, float top_w, float total, float extra)
{
    const float by = total == 0.f ? 0.f : 1.f / total;
    const float by_w = by * (KV_NORM / W_UP) * kv_ex2(top_w - top);
    kv_hadamard(y, l8);
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = total != total ? total : y[i] * by_w;
    if (l8 == 0) y[0] = fmaf(extra * by, 128.f * KV_NORM, y[0]);             // the transform of a row of ones is 128 in its first place
}

// What a row has got from the tokens that its group shares (gbs_kv_shared_attention): as in a partial result, its sums and then m, the total,
// the sum of p mid, and M, with totals that count a token of weight 1 as 1 in both kernels.
constexpr int KV_PREFIX_ROW = GBS_KV_PREFIX_ROW;
__device__ __forceinline__ float* kv_prefix_row(const gbs_kv_attn& A, const KvSeg& s, int token, int head)
{
    return A.prefix + ((long long)(s.e.first + token) * A.n_heads + head) * KV_PREFIX_ROW;
}
// sums of a row in the layout of kv_hadamard
__device__ __forceinline__ void kv_leave_prefix(float* to, const float y[16], int l8, float top, float top_w, float total, float extra)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<float4*>(to + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
    if (l8 == 0) *reinterpret_cast<float4*>(to + 128) = make_float4(top, total, extra, top_w);
}
__device__ __forceinline__ void kv_add_prefix(const float* from, float y[16], int l8, float& top, float& top_w, float& total, float& extra)
{
    const float4 x = *reinterpret_cast<const float4*>(from + 128);
    const float t = fmaxf(top, x.x), t_w = fmaxf(top_w, x.w);
    const float a = kv_ex2(top - t), b = kv_ex2(x.x - t), a_w = kv_ex2(top_w - t_w), b_w = kv_ex2(x.w - t_w);
    total = fmaf(x.y, b, total * a);
    extra = fmaf(x.z, b, extra * a);
    top = t;
    top_w = t_w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(from + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1));
        y[4 * q] = fmaf(v.x, b_w, y[4 * q] * a_w);
        y[4 * q + 1] = fmaf(v.y, b_w, y[4 * q + 1] * a_w);
        y[4 * q + 2] = fmaf(v.z, b_w, y[4 * q + 2] * a_w);
        y[4 * q + 3] = fmaf(v.w, b_w, y[4 * q + 3] * a_w);
    }
}

// row of a tile -> token of the item and query head
__device__ __forceinline__ void kv_row_of(const gbs_kv_attn& A, const KvSeg& s, int row, int& token, int& head)
{
    const int r = s.e.row0 + row;
    token = A.by_group(r);
    head = s.head * A.group + (r - token * A.group);
}

// The number of the block of the kernel before that started the i-th segment that several blocks share, asked by a whole warp; -1: there are fewer.
__device__ __forceinline__ int kv_start_of(const KvAttnArgs& P, int i)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int b0 = 0; b0 < P.blocks; b0 += 128) {
        unsigned which[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) which[k] = b0 + 32 * k + lane < P.blocks ? P.joins[b0 + 32 * k + lane].blocks : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            which[k] = __ballot_sync(0xffffffffu, which[k] != 0);
            const bool here = (which[k] >> lane & 1) && before + __popc(which[k] & ((1u << lane) - 1)) == i;
            const unsigned found = __ballot_sync(0xffffffffu, here);
            if (found != 0) return b0 + 32 * k + __ffs(found) - 1;
            before += __popc(which[k]);
        }
    }
    return -1;
}

// The segments that several blocks share, a warp a row, eight rows a block of this kernel.  Block b joins the one that starts in block b of the kernel before, or, where there
// are far fewer of them than blocks (FEW), the b-th of them: a block that only finds out that there is nothing for it still takes a place for a microsecond, of
// the 4700 that 148 blocks with 256 rows need.  Then the first pieces' sums are also fetched while their weights are found.  17 pieces of 2048 rows: 7.5 us instead of 10.6; with many
// segments the registers for that cost more warps than it gives (44 000 rows 15 us, 23 that way).  The pieces' weights come first, a
// lane a piece, so that their sums can be fetched many at a time: up to a few dozen pieces of a long sequence are as many trips to memory otherwise.
template <int ROWS, int PART, bool FEW>
__global__ __launch_bounds__(256) void k_kv_attn_join(const __grid_constant__ KvAttnArgs P)
{
    constexpr int PIECE = KV_PART<ROWS>;
    __shared__ float full[8][128];
    kv_wait_before();
    kv_let_next();
    const int start = FEW ? kv_start_of(P, blockIdx.x) : (int)blockIdx.x;
    if (start < 0) return;
    const KvJoin j = P.joins[start];
    if (j.blocks == 0) return;
    const gbs_kv_attn& A = P.a;
    const int row = 8 * blockIdx.y + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    // piece b's sums: the first block's last segment, the others' first
    const float* first = P.parts + ((long long)start * 2 + 1) * PIECE;
    const auto piece = [&](int b) { return b == 0 ? first : first + (long long)(2 * b - 1) * PIECE; };
    constexpr int AHEAD = FEW ? 8 : 0;
    float4 ahead[FEW ? AHEAD : 1];
#pragma unroll
    for (int b = 0; b < AHEAD; ++b)
        if (b < j.blocks) ahead[b] = *reinterpret_cast<const float4*>(piece(b) + row * 128 + 4 * lane);
    float top = NONE, top_w = NONE;
    for (int b = lane; b < j.blocks; b += 32) {
        top = fmaxf(top, piece(b)[ROWS * 128 + row]);
        top_w = fmaxf(top_w, piece(b)[ROWS * 128 + 3 * ROWS + row]);
    }
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, h));
        top_w = fmaxf(top_w, __shfl_xor_sync(0xffffffffu, top_w, h));
    }
    float total = 0.f, extra = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int b0 = 0; b0 < j.blocks; b0 += 32) {
        const int n = min(32, j.blocks - b0);
        float weight = 0.f;
        if (lane < n) {
            const float* x = piece(b0 + lane) + ROWS * 128 + row;
            const float keep = kv_ex2(x[0] - top);
            weight = kv_ex2(x[3 * ROWS] - top_w);
            total = fmaf(x[ROWS], keep, total);
            extra = fmaf(x[2 * ROWS], keep, extra);
        }
        const auto add = [&](const float4& x, int b) {
            const float by = __shfl_sync(0xffffffffu, weight, b);
            sum.x = fmaf(x.x, by, sum.x);
            sum.y = fmaf(x.y, by, sum.y);
            sum.z = fmaf(x.z, by, sum.z);
            sum.w = fmaf(x.w, by, sum.w);
        };
        if (b0 == 0)
#pragma unroll
            for (int b = 0; b < AHEAD; ++b)
                if (b < n) add(ahead[b], b);
#pragma unroll 8
        for (int b = b0 == 0 ? AHEAD : 0; b < n; ++b) add(*reinterpret_cast<const float4*>(piece(b0 + b) + row * 128 + 4 * lane), b);
    }
#pragma unroll
    for (int h = 16; h; h >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, h);
        extra += __shfl_xor_sync(0xffffffffu, extra, h);
    }
    *reinterpret_cast<float4*>(&full[row & 7][4 * lane]) = sum;
    __syncwarp();
    KvSeg s;
    s.index = j.index;
    s.head = j.head;
    s.e = kv_entry<PART>(A, P.line, j.index);
    const int l8 = lane & 7;                             // the four groups of eight lanes do the same; the first one writes
    float y[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = full[row & 7][8 * l8 + i];
        y[8 + i] = full[row & 7][64 + 8 * l8 + i];
    }
    if (PART != KV_WHOLE) {
        top -= KV_TOTAL_LOG<ROWS>;
        top_w -= KV_TOTAL_LOG<ROWS>;
    }
    int token, head;
    if (PART == KV_PREFIX) {
        if (s.e.row0 + row >= s.e.rows || lane >= 8) return;
        kv_row_of(A, s, row, token, head);
        kv_leave_prefix(kv_prefix_row(A, s, token, head), y, l8, top, top_w, total, extra);
        return;
    }
    if (PART == KV_OWN && s.e.lo > 0 && s.e.row0 + row < s.e.rows) {
        kv_row_of(A, s, row, token, head);
        kv_add_prefix(kv_prefix_row(A, s, token, head), y, l8, top, top_w, total, extra);
        __syncwarp();
    }
    kv_finish(y, l8, top, top_w, total, extra);
    if (s.e.row0 + row >= s.e.rows || lane >= 8) return;
    kv_row_of(A, s, row, token, head);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + (s.e.first + token) * A.out_token + head * A.out_head;
    if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
    if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
}

}  // namespace
