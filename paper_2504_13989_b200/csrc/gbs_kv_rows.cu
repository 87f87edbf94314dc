// Rows into and out of the paged KV cache (gbs_kv_append, gbs_kv_read).
//
// Eight lanes share a row, so that a warp's loads and stores are 16-byte pieces of four rows: four stages of H_128 in registers, three
// over lanes.  Rows of a token (its heads' keys and values) are neighbours, and so are what they write: the cache's pages are far apart
// only from token to token.
#include "gbs_kv.cuh"

namespace {

constexpr int THREADS = 128, ROWS = THREADS / 8;   // rows of a block

struct RowArgs {
    gbs_kv_view c;
    const int *seqs, *cu;
    int n_items;
    unsigned n_rows, rows_per_token;               // rows: (token, head, key or value)
    int d;
    float c_scale, c_inv, alpha;
    const __nv_bfloat16 *k, *v;
    long long token_stride, head_stride;
    __nv_bfloat16 *k_out, *v_out;
};

// where a row lies in the pool: its codes and its scale(s); null where the token has no place
struct Place {
    unsigned char* codes;
    float* scales;
};

template <bool ASYM>
__device__ __forceinline__ Place place_of(const RowArgs& A, unsigned row, unsigned& token, unsigned& head, bool& value)
{
    // a warp's four rows belong to one token, or to two or more where a token has fewer rows
    token = row / A.rows_per_token;
    const unsigned in = row - token * A.rows_per_token;
    head = in >> 1;
    value = in & 1;
    int item = (int)token, first = (int)token, count = 1;
    if (A.cu) {
        const int t0 = __shfl_sync(0xffffffffu, (int)token, 0), t1 = __shfl_sync(0xffffffffu, (int)token, 31);
        item = -1;
        for (int t = t0; t <= t1; ++t) {
            const int i = kv_item_of(A.cu, A.n_items, t);
            if ((int)token == t) item = i;
        }
    }
    Place p = {nullptr, nullptr};
    if (row >= A.n_rows || item >= A.n_items) return p;
    if (A.cu) {
        first = A.cu[item];
        count = A.cu[item + 1] - first;
    }
    const int seq = kv_sequence(A.c, A.seqs, item);
    if (seq < 0) return p;
    const int length = kv_length(A.c, seq), pos = length - count + ((int)token - first);
    if (pos < 0 || pos >= length) return p;
    const int page = kv_page(A.c, seq, pos);
    if (page < 0) return p;
    unsigned char* block = kv_block(A.c, page, (int)head);
    const int ps = 1 << A.c.page_log, slot = pos & (ps - 1);
    p.codes = block + (value ? ps * KV_ROW : 0) + slot * KV_ROW;
    p.scales = reinterpret_cast<float*>(block + 2 * ps * KV_ROW) + ((value ? ps : 0) + slot) * (ASYM ? 2 : 1);
    return p;
}

__device__ __forceinline__ float max8(float x)
{
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, h));
    return x;
}

// eight codes, lowest coordinate in the lowest nibble
__device__ __forceinline__ unsigned pack8(const float y[8], float inv, float low, float high)
{
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int q = __float2int_rn(fminf(fmaxf(y[i] * inv, low), high));
        w |= (unsigned)(q & 15) << (4 * i);
    }
    return w;
}

constexpr float TINY = 1e-30f, UP = 1.2379400392853803e27f;     // 2^90

template <bool ASYM>
__global__ __launch_bounds__(THREADS) void k_kv_append(const __grid_constant__ RowArgs A)
{
    kv_wait_before();
    kv_let_next();
    const unsigned row = blockIdx.x * ROWS + (threadIdx.x >> 3);
    const int l8 = threadIdx.x & 7;
    unsigned token, head;
    bool value;
    const Place p = place_of<ASYM>(A, row, token, head, value);
    float y[16];
    uint4 a = make_uint4(0, 0, 0, 0), b = a;
    if (p.codes) {
        const __nv_bfloat16* x = (value ? A.v : A.k) + (long long)token * A.token_stride + (long long)head * A.head_stride;
        if (8 * l8 < A.d) a = *reinterpret_cast<const uint4*>(x + 8 * l8);
        if (64 + 8 * l8 < A.d) b = *reinterpret_cast<const uint4*>(x + 64 + 8 * l8);
    }
    kv_unpack_bf16(a, y);
    kv_unpack_bf16(b, y + 8);
    kv_hadamard(y, l8);
    // rows of the smallest numbers: their quotients are taken at 2^90 times the size
    if (ASYM) {
        float mn = y[0], mx = y[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) {
            mn = fminf(mn, y[i]);
            mx = fmaxf(mx, y[i]);
        }
        mx = max8(mx);
        mn = -max8(-mn);
        const float lo = A.alpha * mn, hi = A.alpha * mx, up = hi - lo < TINY ? UP : 1.f;
        const float span = (hi - lo) * up, inv = span > 0.f ? 15.f / span : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = (y[i] - lo) * up;
        if (p.codes) {
            *reinterpret_cast<unsigned*>(p.codes + 4 * l8) = pack8(y, inv, 0.f, 15.f);
            *reinterpret_cast<unsigned*>(p.codes + 32 + 4 * l8) = pack8(y + 8, inv, 0.f, 15.f);
            if (l8 == 0) *reinterpret_cast<float2*>(p.scales) = make_float2((hi - lo) * (KV_NORM / 15.f), lo * KV_NORM);
        }
    } else {
        float m = fabsf(y[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, fabsf(y[i]));
        m = max8(m);
        const float up = m < TINY ? UP : 1.f, inv = m > 0.f ? A.c_inv / (m * up) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] *= up;
        if (p.codes) {
            *reinterpret_cast<unsigned*>(p.codes + 4 * l8) = pack8(y, inv, -7.f, 7.f);
            *reinterpret_cast<unsigned*>(p.codes + 32 + 4 * l8) = pack8(y + 8, inv, -7.f, 7.f);
            if (l8 == 0) *p.scales = A.c_scale * m;
        }
    }
}

template <bool ASYM>
__global__ __launch_bounds__(THREADS) void k_kv_read(const __grid_constant__ RowArgs A)
{
    kv_wait_before();
    kv_let_next();
    const unsigned row = blockIdx.x * ROWS + (threadIdx.x >> 3);
    const int l8 = threadIdx.x & 7;
    unsigned token, head;
    bool value;
    const Place p = place_of<ASYM>(A, row, token, head, value);
    unsigned w[2] = {0, 0};
    float scale = 0.f, lo = 0.f;
    if (p.codes) {
        w[0] = *reinterpret_cast<const unsigned*>(p.codes + 4 * l8);
        w[1] = *reinterpret_cast<const unsigned*>(p.codes + 32 + 4 * l8);
        if (ASYM) {
            const float2 s = *reinterpret_cast<const float2*>(p.scales);
            scale = s.x;
            lo = s.y;
        } else scale = *p.scales;
    }
    // the codes are rotated exactly; the transform of a row of ones is sqrt(128) in its first coordinate, once normalised
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = (int)(w[i >> 3] >> (4 * (i & 7))) & 15;
        y[i] = (float)(ASYM ? q : (q ^ 8) - 8);
    }
    kv_hadamard(y, l8);
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] *= scale * KV_NORM;
    if (ASYM && l8 == 0) y[0] = fmaf(lo, 11.313708498984761f, y[0]);
    // rows behind the last item stay as they are, rows without a place become 0
    if (row >= A.n_rows || (A.cu && (int)token >= A.cu[A.n_items])) return;
    __nv_bfloat16* out = (value ? A.v_out : A.k_out) + ((long long)token * A.c.heads + head) * A.d;
    if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
    if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
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
    A.c_inv = p->c_inv;
    A.alpha = p->alpha;
    return A;
}

}  // namespace

int gbs_kv_append_launch(const gbs_plan* p, const gbs_kv_view& c, const int* seqs, const int* cu, int n_items, int64_t n_tokens, const void* k,
                         const void* v, int64_t token_stride, int64_t head_stride, cudaStream_t stream)
{
    RowArgs A = row_args(p, c, seqs, cu, n_items, n_tokens);
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
