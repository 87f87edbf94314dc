// Rows into and out of the paged KV cache (gbs_kv_append, gbs_kv_read).
//
// A warp takes 16 rows.  H_128 is a product of seven butterfly stages, one per bit of the coordinate; four of them are one H_16, which the
// matrix unit does (16 rows x 16 coordinates times +-1, products exact, fp32 sums), the other three are additions between registers of a
// thread.  Which bits go where follows from how rows lie in memory: thread (g, t) of a warp (g = lane / 4, t = lane % 4) holds, of rows
// g and g + 8, coordinates 8 (t + 4 j) .. + 7 for j = 0 .. 3, that is 16-byte pieces of 16-bit rows and 4-byte pieces of codes, four lanes next to each
// other.  Bits 3 and 4 (t) lie across lanes and have to go to the matrix unit, with two of the three bits below; what is left, the third
// one and j, is in registers.  The result has the layout of the operand, so no number moves between lanes.
// Seven stages over eight lanes a row, three of them by shuffles, took 119 and 85 instructions a row and warp (write and read) instead of 59 and 52:
// 14000 tokens x 8 heads written and read back in 62.7 us instead of 44.
// The bytes (130 MB) would take 20 us.  Issue slots are 57 % used; the rest is waiting for a warp's 16 rows, which nothing overlaps.
// Reading back, the codes go in as fp16, and everything up to the scale is exact.
#include <cuda_fp16.h>

#include "gbs_kv.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int THREADS = 128, ROWS = THREADS / 2;   // rows of a block

struct RowArgs {
    gbs_kv_view c;
    const int *seqs, *cu, *status;                 // status: of an extend; items that it refused have no place (null: all have)
    int n_items;
    unsigned n_rows, rows_per_token;               // rows: (token, head, key or value)
    int d;
    float c_scale, c_half, alpha;
    const __nv_bfloat16 *k, *v;
    long long token_stride, head_stride;
    __nv_bfloat16 *k_out, *v_out;
};

// where the row of a lane lies in the pool: its codes and its scale(s); null where the token has no place
struct Place {
    unsigned char* codes;
    float* scales;
};
// A token's place: its page (head 0; null: none) and its slot there.
struct TokenPlace {
    unsigned char* page;
    int slot;
};

// Places of a warp's tokens, first .. last (at most 32): lane i finds token first + i, so that the chain of lookups (item, sequence,
// length, page) is gone through once for all of the warp's rows.
__device__ __forceinline__ TokenPlace look_up(const RowArgs& A, int first, int last)
{
    const int lane = threadIdx.x & 31, token = first + lane;
    TokenPlace p = {nullptr, 0};
    int item = token, from = token, count = 1;
    if (A.cu) {
        if (first == last) item = kv_item_of(A.cu, A.n_items, first);
        else {
            int lo = 0, hi = A.n_items;                  // how many of cu[1 .. n] are <= token
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (A.cu[mid + 1] <= token) lo = mid + 1;
                else hi = mid;
            }
            item = lo;
        }
    }
    if (token > last || (unsigned)item >= (unsigned)A.n_items) return p;
    if (A.cu) {
        from = A.cu[item];
        count = A.cu[item + 1] - from;
        if (token < from) return p;                      // before the first item
    }
    const int seq = kv_sequence(A.c, A.seqs, item);
    if (seq < 0 || (A.status && A.status[item] != GBS_KV_DONE)) return p;
    const int length = kv_length(A.c, seq), pos = length - count + (token - from);
    if (pos < 0 || pos >= length) return p;
    const int page = kv_page(A.c, seq, pos);
    if (page < 0) return p;
    p.page = kv_block(A.c, page, 0);
    p.slot = pos & ((1 << A.c.page_log) - 1);
    return p;
}
__device__ __forceinline__ TokenPlace of_lane(const TokenPlace& p, int lane)
{
    return TokenPlace{reinterpret_cast<unsigned char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(p.page), lane)), __shfl_sync(0xffffffffu, p.slot, lane)};
}
template <bool ASYM>
__device__ __forceinline__ Place place_of(const RowArgs& A, const TokenPlace& t, unsigned head, bool value)
{
    if (!t.page) return Place{nullptr, nullptr};
    unsigned char* block = t.page + (long long)head * A.c.block_bytes;
    const int ps = 1 << A.c.page_log;
    return Place{block + ((value ? ps : 0) + t.slot) * KV_ROW, reinterpret_cast<float*>(block + 2 * ps * KV_ROW) + ((value ? ps : 0) + t.slot) * (ASYM ? 2 : 1)};
}

// the lanes of a row
__device__ __forceinline__ float max4(float x)
{
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}

// c = a b
template <bool HALF>
__device__ __forceinline__ void mma_16(float c[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    if (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// H_128 (unnormalised) of 16 rows.  in[row][j][p]: pairs of row g (g + 8) of coordinates 8 (t + 4 j) .., y[row][8 j + k]: results, coordinate
// 8 (t + 4 j) + k.  bf16 rows: pair p is coordinates 2 p, 2 p + 1 (bit 0 in the pair); codes in fp16: p, p + 4 (bit 2 in the pair).
// A step of the matrix unit contracts the pair's bit, one more bit of p, and t; its 16 columns are column bit 0 = the pair's bit of the
// result for bf16 (bit 0 either way), the columns' halves the other one, and t again.  The third bit of p and j are added up afterwards.
template <bool HALF>
__device__ __forceinline__ void rotate16(const unsigned in[2][4][4], float y[2][32], int lane)
{
    const int t = lane & 3, n = lane >> 2;               // the operand's column is 2 t' + e
    constexpr unsigned ONE = HALF ? 0x3c00u : 0x3f80u;
    const unsigned sign = (__popc(t & (n >> 1)) & 1) ? 0x80008000u : 0u, odd = n & 1;
    const unsigned same = (ONE | ONE << 16) ^ sign, flip = same ^ 0x80000000u, minus = same ^ 0x80008000u;
    // bf16: k = (t, bit 0 in the pair, bit 1 second register), columns (t', bit 0 = e, bit 1 = half)
    // fp16: k = (t, bit 2 in the pair, bit 0 second register), columns (t', bit 0 = e, bit 2 = half)
    const unsigned b00 = HALF ? same : odd ? flip : same, b01 = HALF ? (odd ? minus : same) : b00;
    const unsigned b10 = HALF ? flip : b00, b11 = HALF ? (odd ? flip ^ 0x80008000u : flip) : b00 ^ 0x80008000u;
    float c[4][2][2][4];                                 // [j][step: bit 2 (bf16), bit 1 (fp16)][half of the columns]
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            mma_16<HALF>(c[j][s][0], in[0][j][2 * s], in[1][j][2 * s], in[0][j][2 * s + 1], in[1][j][2 * s + 1], b00, b01);
            mma_16<HALF>(c[j][s][1], in[0][j][2 * s], in[1][j][2 * s], in[0][j][2 * s + 1], in[1][j][2 * s + 1], b10, b11);
        }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v[8];                              // (step, j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = c[i & 3][i >> 2][h][2 * r + e];
#pragma unroll
                for (int k = 1; k < 8; k <<= 1)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if ((i & k) == 0) {
                            const float a = v[i], b = v[i + k];
                            v[i] = a + b;
                            v[i + k] = a - b;
                        }
#pragma unroll
                for (int i = 0; i < 8; ++i) y[r][8 * (i & 3) + (HALF ? e + 4 * h + 2 * (i >> 2) : e + 2 * h + 4 * (i >> 2))] = v[i];
            }
}

// eight codes of numbers w = y a1 + c0 in [0, 1] (which also clips), lowest coordinate in the lowest nibble
template <bool ASYM>
__device__ __forceinline__ unsigned pack8(const float y[8], float a1, float c0)
{
    unsigned r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(y[i]);
    return __byte_perm(quantize4<4, !ASYM>(r, a1, c0), quantize4<4, !ASYM>(r + 4, a1, c0), 0x5410) ^ (ASYM ? 0u : 0x88888888u);
}

constexpr float TINY = 1e-30f, UP = 1.2379400392853803e27f;     // 2^90

// a lane's two rows: g and g + 8 of the warp's 16
struct TwoRows {
    unsigned token[2], head[2];
    bool value[2], there[2];
    Place place[2];
};
__device__ __forceinline__ void name_rows(const RowArgs& A, unsigned row, TwoRows& R)
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const unsigned at = min(row + 8 * r, A.n_rows - 1);
        R.there[r] = row + 8 * r < A.n_rows;
        R.token[r] = at / A.rows_per_token;
        const unsigned in = at - R.token[r] * A.rows_per_token;
        R.head[r] = in >> 1;
        R.value[r] = in & 1;
    }
}
template <bool ASYM>
__device__ __forceinline__ void find_rows(const RowArgs& A, const TokenPlace& places, int first, TwoRows& R)
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const TokenPlace t = of_lane(places, (int)R.token[r] - first);
        R.place[r] = R.there[r] ? place_of<ASYM>(A, t, R.head[r], R.value[r]) : Place{nullptr, nullptr};
    }
}

template <bool ASYM>
__global__ __launch_bounds__(THREADS) void k_kv_append(const __grid_constant__ RowArgs A)
{
    kv_wait_before();
    kv_let_next();
    const int lane = threadIdx.x & 31, t = lane & 3;
    const unsigned row0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * 16u;
    if (row0 >= A.n_rows) return;
    const int first = (int)(row0 / A.rows_per_token), last = (int)(min(row0 + 15u, A.n_rows - 1) / A.rows_per_token);
    TwoRows R;
    name_rows(A, row0 + (lane >> 2), R);
    unsigned in[2][4][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const __nv_bfloat16* x = (R.value[r] ? A.v : A.k) + (long long)R.token[r] * A.token_stride + (long long)R.head[r] * A.head_stride;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (8 * (t + 4 * j) < A.d) q = *reinterpret_cast<const uint4*>(x + 8 * (t + 4 * j));
            in[r][j][0] = q.x; in[r][j][1] = q.y; in[r][j][2] = q.z; in[r][j][3] = q.w;
        }
    }
    find_rows<ASYM>(A, look_up(A, first, last), first, R);      // while the rows are on their way
    float y[2][32];
    rotate16<false>(in, y, lane);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        // a number w in [0, 1] of a coordinate is y a1 + c0; rows of the smallest numbers are taken at 2^90 times their size
        float a1, c0 = 0.5f, scale, lo = 0.f, up = 1.f;
        if (ASYM) {
            float mn = y[r][0], mx = y[r][0];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
                mn = min3(y[r][k], y[r][k + 1], mn);
                mx = max3(y[r][k], y[r][k + 1], mx);
            }
            mx = max4(mx);
            mn = -max4(-mn);
            lo = A.alpha * mn;
            const float span = A.alpha * mx - lo;
            if (span < TINY) up = UP;
            scale = span * (KV_NORM / 15.f);
            a1 = span > 0.f ? 1.f / (span * up) : 0.f;
            c0 = -(lo * up) * a1;
            lo *= KV_NORM;
        } else {
            float m = 0.f;
#pragma unroll
            for (int k = 0; k < 32; k += 2) m = max3(fabsf(y[r][k]), fabsf(y[r][k + 1]), m);
            m = max4(m);
            if (m < TINY) up = UP;
            scale = A.c_scale * m;
            // every coordinate of a row with a NaN is one, and the maximum passes over them
            if (y[r][0] != y[r][0]) scale = y[r][0];
            a1 = m > 0.f ? A.c_half / (m * up) : 0.f;
        }
        if (up != 1.f) {
#pragma unroll
            for (int k = 0; k < 32; ++k) y[r][k] *= up;
        }
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack8<ASYM>(&y[r][8 * j], a1, c0);
        if (R.place[r].codes) {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<unsigned*>(R.place[r].codes + 4 * (t + 4 * j)) = w[j];
            if (t == 0) {
                if (ASYM) *reinterpret_cast<float2*>(R.place[r].scales) = make_float2(scale, lo);
                else *R.place[r].scales = scale;
            }
        }
    }
}

__device__ __forceinline__ unsigned as_u(__half2 x) { return *reinterpret_cast<unsigned*>(&x); }
__device__ __forceinline__ __half2 as_h(unsigned x) { return *reinterpret_cast<__half2*>(&x); }

template <bool ASYM>
__global__ __launch_bounds__(THREADS) void k_kv_read(const __grid_constant__ RowArgs A)
{
    kv_wait_before();
    kv_let_next();
    const int lane = threadIdx.x & 31, t = lane & 3;
    const int end = A.cu ? A.cu[A.n_items] : 0x7fffffff;
    const unsigned row0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * 16u;
    if (row0 >= A.n_rows) return;
    const int first = (int)(row0 / A.rows_per_token), last = (int)(min(row0 + 15u, A.n_rows - 1) / A.rows_per_token);
    const TokenPlace places = look_up(A, first, last);
    TwoRows R;
    name_rows(A, row0 + (lane >> 2), R);
    find_rows<ASYM>(A, places, first, R);
    unsigned in[2][4][4];
    float scale[2] = {0.f, 0.f}, lo[2] = {0.f, 0.f};
    unsigned w[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[r][j] = R.place[r].codes ? *reinterpret_cast<const unsigned*>(R.place[r].codes + 4 * (t + 4 * j)) : 0u;
        if (R.place[r].codes) {
            if (ASYM) {
                const float2 s = *reinterpret_cast<const float2*>(R.place[r].scales);
                scale[r] = s.x;
                lo[r] = s.y;
            } else scale[r] = *R.place[r].scales;
        }
    }
    // pairs (coordinate k, k + 4) of each eight: a nibble in the mantissa of 1024, which is subtracted again
    constexpr unsigned LOW = ASYM ? 0x64006400u : 0x64086408u, HIGH = ASYM ? 0x64006400u : 0x64806480u;
    const __half2 off = __float2half2_rn(ASYM ? 1024.f : 1032.f), off16 = __float2half2_rn(ASYM ? -64.f : -72.f), sixteenth = __float2half2_rn(0.0625f);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned x = w[r][j], x8 = x >> 8;
            in[r][j][0] = as_u(__hsub2(as_h((x & 0x000f000fu) ^ LOW), off));
            in[r][j][1] = as_u(__hfma2(as_h((x & 0x00f000f0u) ^ HIGH), sixteenth, off16));
            in[r][j][2] = as_u(__hsub2(as_h((x8 & 0x000f000fu) ^ LOW), off));
            in[r][j][3] = as_u(__hfma2(as_h((x8 & 0x00f000f0u) ^ HIGH), sixteenth, off16));
        }
    float y[2][32];
    rotate16<true>(in, y, lane);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        // rows behind the last item stay as they are, rows without a place become 0
        if (!R.there[r] || (int)R.token[r] >= end) continue;
        const float by = scale[r] * KV_NORM;
#pragma unroll
        for (int k = 0; k < 32; ++k) y[r][k] *= by;
        // the transform of a row of ones is sqrt(128) in its first coordinate, once normalised
        if (ASYM && t == 0) y[r][0] = fmaf(lo[r], 11.313708498984761f, y[r][0]);
        __nv_bfloat16* out = (R.value[r] ? A.v_out : A.k_out) + ((long long)R.token[r] * A.c.heads + R.head[r]) * A.d;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (8 * (t + 4 * j) < A.d) *reinterpret_cast<uint4*>(out + 8 * (t + 4 * j)) = kv_pack_bf16(&y[r][8 * j]);
    }
}

RowArgs row_args(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, const int* cu, int n_items, int64_t n_tokens)
{
    RowArgs A = {};
    A.c = c;
    A.seqs = seqs;
    A.cu = cu;
    A.n_items = n_items;
    A.rows_per_token = 2u * c.heads;
    A.n_rows = (unsigned)(n_tokens * A.rows_per_token);
    A.d = p->d;
    A.c_scale = p->c_scale;
    A.c_half = (float)(0.5 / (double)p->alpha);
    A.alpha = p->alpha;
    return A;
}

}  // namespace

int gbs_kv_append_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, const int* cu, int n_items, int64_t n_tokens, const void* k,
                         const void* v, int64_t token_stride, int64_t head_stride, const int* status, cudaStream_t stream)
{
    RowArgs A = row_args(p, c, seqs, cu, n_items, n_tokens);
    A.status = status;
    A.k = static_cast<const __nv_bfloat16*>(k);
    A.v = static_cast<const __nv_bfloat16*>(v);
    A.token_stride = token_stride;
    A.head_stride = head_stride;
    return gbs_kv_launch(p, p->asym ? k_kv_append<true> : k_kv_append<false>, dim3((A.n_rows + ROWS - 1) / ROWS), THREADS, 0, stream, A);
}

int gbs_kv_read_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, const int* cu, int n_items, int64_t n_tokens, void* k_out,
                       void* v_out, cudaStream_t stream)
{
    RowArgs A = row_args(p, c, seqs, cu, n_items, n_tokens);
    A.k_out = static_cast<__nv_bfloat16*>(k_out);
    A.v_out = static_cast<__nv_bfloat16*>(v_out);
    return gbs_kv_launch(p, p->asym ? k_kv_read<true> : k_kv_read<false>, dim3((A.n_rows + ROWS - 1) / ROWS), THREADS, 0, stream, A);
}
