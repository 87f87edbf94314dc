// Attention over the paged KV cache for prompts and chunks of them (gbs_kv_attention, more than 16 query rows of an item and KV head), on
// tcgen05: tiles of 128 rows (tokens x query heads of a KV head) by 128 cached tokens.
//
// The mathematics is that of gbs_kv_attn.cu: codes enter the matrix unit as they are (exact in fp16), scales stay outside.
//     S = Q C_k^T (fp16, fp32 sums),  z = S Delta_k f + log2 Delta_v,  w = 2^(z - M + 6),  O += w C_v,  l += w / Delta_v.
// With log2 Delta_v inside the exponent one running maximum M (of z) serves both the weights' range in fp16 and the softmax; a row with zero
// values alone has codes 0, and takes the largest scale next to it.  f is the row's factor (its power of two, the softmax scale).
//
// Warps 0-3: softmax, a thread a row.  Warps 4-7: codes to fp16, a thread a cached token; they fetch the next tile's codes into
// registers while this one's are worked on.  Warp 4 also issues the MMAs: a ninth warp would cost all of them 32 registers each.  Scores and weights share 128 columns of tensor memory (a thread's
// fp16 weights overwrite scores it has read), the sums take 128 more, so two blocks run on an SM and fill each other's gaps.
// The work per tile and SM: 2 x 512 cycles of MMA, 1024 of ex2; what bounds it is REPLACE.
#include "gbs_kv_attn.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int ROWS = 128, UNIT = 128;
constexpr int THREADS = 256;
constexpr int BLOCKS_PER_SM = 2;
constexpr int PART = KV_PART<ROWS>;
constexpr float MOVE = 8.f;                          // M moves when a score is so much (log2) above it
constexpr unsigned O_COL = 128, TMEM_COLS = 256;

struct Smem {
    unsigned char q[ROWS * 256];                     // fp16, K-major, two blocks of 64 coordinates, 128-byte swizzle
    unsigned char k[UNIT * 256];                     // the same; at a segment's end k and v hold its sums in fp32
    unsigned char v[UNIT * 256];                     // N-major for the second product: the same bytes
    float ks[2][UNIT], lv[2][UNIT], rv[2][UNIT], kl[2][UNIT], vl[2][UNIT];       // of tile i in [i & 1]: Delta_k, log2 Delta_v, 1 / Delta_v, lo
    float factor[ROWS], qsum[ROWS];
    float m[ROWS], l[ROWS], add[ROWS];
    unsigned long long kfull, kfree, vfull, vfree, sfull, pfull;
    KvSeg seg;
    long long share[THREADS / 32];
    unsigned tmem;
    int abort;
};

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 both(float x) { return pk(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ void tmem_ld_wait16(unsigned r[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
          "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// byte of a 16-byte piece (8 coordinates) of a row in a tile
__device__ __forceinline__ unsigned piece_at(int row, int piece)
{
    return (unsigned)(piece >> 3) * (128 * 128) + (unsigned)(row >> 3) * 1024 + (unsigned)(row & 7) * 128 + (unsigned)(((piece & 7) ^ (row & 7)) << 4);
}
// byte of a 16-byte piece (4 coordinates) of a row of sums
__device__ __forceinline__ unsigned sum_at(int row, int piece) { return (unsigned)row * 512 + (unsigned)((piece ^ (row & 31)) << 4); }

// A cached token's codes and scales on their way through registers.
struct Token {
    uint4 k[4], v[4];
    float ks, kl, vs, vl;
    bool ok;
};

__device__ __forceinline__ const unsigned char* find(const gbs_kv_attn& A, const KvSeg& s, int tok, int page)
{
    if (tok < s.e.lo || tok >= s.e.hi || (unsigned)page >= (unsigned)A.c.n_pages) return nullptr;
    return kv_block(A.c, page, s.head);
}
template <bool ASYM>
__device__ __forceinline__ void load_k(Token& x, const unsigned char* block, int slot, int ps)
{
    x.ok = block != nullptr;
    x.ks = x.kl = x.vl = 0.f;
    x.vs = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.k[i] = make_uint4(0, 0, 0, 0);
    if (!block) return;
    const uint4* c = reinterpret_cast<const uint4*>(block + slot * KV_ROW);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.k[i] = c[i];
    const float* sc = reinterpret_cast<const float*>(block + 2 * ps * KV_ROW);
    if (ASYM) {
        const float2 a = reinterpret_cast<const float2*>(sc)[slot], b = reinterpret_cast<const float2*>(sc)[ps + slot];
        x.ks = a.x; x.kl = a.y; x.vs = b.x; x.vl = b.y;
    } else {
        x.ks = sc[slot];
        x.vs = sc[ps + slot];
    }
}
__device__ __forceinline__ void load_v(Token& x, const unsigned char* block, int slot, int ps)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = make_uint4(0, 0, 0, 0);
    if (!block) return;
    const uint4* c = reinterpret_cast<const uint4*>(block + (ps + slot) * KV_ROW);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = c[i];
}
// A word's 8 coordinates stand in the order 0, 4, 1, 5, 2, 6, 3, 7, in the queries as well; the results' columns are put back at the end.
template <bool ASYM>
__device__ __forceinline__ void store_codes(unsigned char* tile, int row, const uint4 c[4])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint4 q = c[i >> 2];
        const unsigned w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
        unsigned h[4];
        kv_codes_f16<ASYM>(w, h);
        *reinterpret_cast<uint4*>(tile + piece_at(row, i)) = make_uint4(h[0], h[1], h[2], h[3]);
    }
}

template <bool ASYM>
__global__ __launch_bounds__(THREADS, BLOCKS_PER_SM) void k_tc_kvattn(const __grid_constant__ KvAttnArgs P)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, w = warp_index();
    if (tid == 0) {
        S.abort = 0;
        mbar_init(&S.kfull, 128);
        mbar_init(&S.kfree, 1);
        mbar_init(&S.vfull, 128);
        mbar_init(&S.vfree, 1);
        mbar_init(&S.sfull, 1);
        mbar_init(&S.pfull, 128);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == 4) tmem_alloc(&S.tmem, TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = S.tmem;
    kv_wait_before();
    kv_let_next();

    const int places = kv_share<THREADS>(A, P.line, &S.seg, S.share);
    KvSeg seg = S.seg;
    if (tid == 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};

    const int ps_log = A.c.page_log, ps = 1 << ps_log;
    unsigned it = 0;                                         // tiles so far, by which the barriers' phases go
    for (bool more = places > 0; more;) {
        const KvPiece piece = kv_piece(P.line, seg, places);
        const int n = piece.n, tok0 = (seg.e.lo / UNIT + piece.skip) * UNIT;
        if (n <= 0) break;                                   // the block's last places are in front of a segment's units

        // ---- query rows: eight lanes a row, 32 rows at a time ----
        Token x;
        const unsigned char* block = nullptr;
        int page = -1;
        if (w >= 4) {
            const int tok = tok0 + tid - 128;
            const int* row = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            block = find(A, seg, tok, tok < seg.e.hi ? row[tok >> ps_log] : -1);
            load_k<ASYM>(x, block, tok & (ps - 1), ps);
            load_v(x, block, tok & (ps - 1), ps);
            page = tok + UNIT < seg.e.hi ? row[(tok + UNIT) >> ps_log] : -1;
        }
        {
            const int l8 = tid & 7;
            uint4 raw[4][2];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 32 * r + (tid >> 3);
                raw[r][0] = raw[r][1] = make_uint4(0, 0, 0, 0);
                if (seg.e.row0 + row < seg.e.rows) {
                    int token, head;
                    kv_row_of(A, seg, row, token, head);
                    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(A.q) + (seg.e.first + token) * A.q_token + head * A.q_head;
                    if (8 * l8 < A.d) raw[r][0] = *reinterpret_cast<const uint4*>(q + 8 * l8);
                    if (64 + 8 * l8 < A.d) raw[r][1] = *reinterpret_cast<const uint4*>(q + 64 + 8 * l8);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 32 * r + (tid >> 3);
                float y[16];
                kv_unpack_bf16(raw[r][0], y);
                kv_unpack_bf16(raw[r][1], y + 8);
                kv_hadamard(y, l8);
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(y[i]));
#pragma unroll
                for (int h = 1; h < 8; h <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, h));
                // the largest coordinate of a row just below 2^8: far from fp16's smallest numbers.  2^(134 - e) and its inverse
                const int e = min(max((int)(__float_as_uint(m) >> 23), 8), 252);
                const float down = __uint_as_float((unsigned)(261 - e) << 23), up = __uint_as_float((unsigned)(e - 7) << 23);
                float sum = 0.f;
                __half h[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    h[i] = __float2half_rn(y[i] * down);
                    sum += __half2float(h[i]);
                }
#pragma unroll
                for (int k = 1; k < 8; k <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const __half* g = h + 8 * half;
                    *reinterpret_cast<uint4*>(S.q + piece_at(row, 8 * half + l8)) =
                        make_uint4(as_u(__halves2half2(g[0], g[4])), as_u(__halves2half2(g[1], g[5])), as_u(__halves2half2(g[2], g[6])), as_u(__halves2half2(g[3], g[7])));
                }
                if (l8 == 0) {
                    S.factor[row] = up * (A.scale * (KV_NORM * 1.4426950408889634f));
                    S.qsum[row] = sum;
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();

        if (w >= 4) {
            // ---- codes to fp16; warp 4: the MMAs as well ----
            constexpr unsigned ID_S = (1u << 4) | ((unsigned)(UNIT >> 3) << 17) | ((unsigned)(ROWS >> 4) << 24);             // fp16, both K-major
            constexpr unsigned ID_O = ID_S | (1u << 16);                                                                    // B N-major
            const unsigned long long qd = smem_desc(smem_u32(S.q), 16, 1024, 2), kd = smem_desc(smem_u32(S.k), 16, 1024, 2),
                                     vd = smem_desc(smem_u32(S.v), 128 * 128, 1024, 2);
            const int me = tid - 128;
            const int* row = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            // the keys of tile i into shared memory, those of tile i + 1 on their way
            auto keys = [&](int i) {
                const unsigned now = it + i;
                const int tok = tok0 + i * UNIT + me, b = now & 1;
                // zero rows take the largest scale next to them; tokens that are not there weigh nothing, and scales that are no
                // numbers make the scores of those that see them none
                float vs = x.vs, near = x.vs;
#pragma unroll
                for (int h = 16; h; h >>= 1) near = fmaxf(near, __shfl_xor_sync(0xffffffffu, near, h));
                const bool wrong = !(fabsf(vs) < INFINITY) || !(fabsf(x.vl) < INFINITY);
                if (vs == 0.f) vs = near > 0.f ? near : 1.f;
                vs = fmaxf(vs, 7.888609052210118e-31f);                          // 2^-100
                const float lv = !x.ok ? -INFINITY : wrong ? NAN : __log2f(vs), rv = x.ok && !wrong ? 1.f / vs : 0.f;
                if (now > 0 && !mbar_wait(&S.abort, &S.kfree, (now + 1) & 1u, P.status, 74)) return false;
                S.ks[b][me] = x.ks;
                S.lv[b][me] = lv;
                S.rv[b][me] = rv;
                if (ASYM) {
                    S.kl[b][me] = x.kl;
                    S.vl[b][me] = wrong ? 0.f : x.vl;
                }
                store_codes<ASYM>(S.k, me, x.k);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(&S.kfull);
                const int next = tok + UNIT;
                block = i + 1 < n ? find(A, seg, next, page) : nullptr;
                page = next + UNIT < seg.e.hi ? row[(next + UNIT) >> ps_log] : -1;
                load_k<ASYM>(x, block, next & (ps - 1), ps);
                return true;
            };
            auto scores = [&](int i) {
                if (w != 4) return true;
                if (!mbar_wait_warp(&S.abort, &S.kfull, (it + i) & 1u, P.status, 71)) return false;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 8; ++k) {                // sixteen coordinates: 32 bytes, four of them in a block of 64
                    const unsigned long long off = (unsigned)((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
                    umma_f16(tmem, qd + off, kd + off, ID_S, k > 0);
                }
                umma_commit(&S.sfull);
                umma_commit(&S.kfree);
                return true;
            };
            bool ok = __all_sync(0xffffffffu, keys(0));
            if (ok) ok = scores(0);
            for (int i = 0; i < n && __all_sync(0xffffffffu, ok); ++i) {
                const unsigned now = it + i;
                const int tok = tok0 + i * UNIT + me;
                if (now > 0 && !mbar_wait(&S.abort, &S.vfree, (now + 1) & 1u, P.status, 75)) ok = false;
                if (!__all_sync(0xffffffffu, ok)) break;
                store_codes<ASYM>(S.v, me, x.v);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(&S.vfull);
                if (i + 1 < n) {
                    const unsigned char* ahead = block;
                    load_v(x, ahead, (tok + UNIT) & (ps - 1), ps);
                    ok = keys(i + 1);
                }
                if (w == 4) {
                    if (!__all_sync(0xffffffffu, ok) || !mbar_wait_warp(&S.abort, &S.vfull, now & 1u, P.status, 72) ||
                        !mbar_wait_warp(&S.abort, &S.pfull, now & 1u, P.status, 73)) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 8; ++k)              // sixteen tokens: two groups of eight rows
                        umma_f16_ts(tmem + O_COL, tmem + 8 * k, vd + (unsigned)((k * 2048) >> 4), ID_O, i > 0 || k > 0);
                    umma_commit(&S.vfree);
                    if (i + 1 < n) ok = scores(i + 1);
                }
            }
        } else {
            // ---- softmax: a thread a row ----
            const unsigned lanes = tmem + ((unsigned)w << 21);
            const bool here = seg.e.row0 + tid < seg.e.rows;
            const int my_token = A.by_group(min(seg.e.row0 + tid, seg.e.rows - 1));
            const int row_lo = kv_row_lo(A, seg.e, my_token), row_hi = here ? kv_row_hi(A, seg.e, my_token) : 0;
            // tokens that every row of the tile sees need no mask
            const int all_lo = kv_row_lo(A, seg.e, A.by_group(min(seg.e.rows, seg.e.row0 + ROWS) - 1)), all_hi = kv_row_hi(A, seg.e, A.by_group(seg.e.row0));
            const float f = S.factor[tid], qs = S.qsum[tid];
            const f32x2 f2 = both(f), qs2 = both(qs);
            float M = NONE;
            f32x2 l2 = both(0.f), add2v = both(0.f);
            bool ok = true;
            for (int i = 0; i < n && ok; ++i) {
                const unsigned now = it + i;
                const int b = now & 1, tok = tok0 + i * UNIT;
                const bool plain = tok >= all_lo && tok + UNIT <= all_hi;
                if (!(ok = mbar_wait_warp(&S.abort, &S.sfull, now & 1u, P.status, 76))) break;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    unsigned r[32];
                    tmem_ld32_issue(lanes + 32 * c, r);
                    tmem_ld_wait(r);
                    const ulonglong2* ks = reinterpret_cast<const ulonglong2*>(&S.ks[b][32 * c]);
                    const ulonglong2* lv = reinterpret_cast<const ulonglong2*>(&S.lv[b][32 * c]);
                    const ulonglong2* kl = reinterpret_cast<const ulonglong2*>(&S.kl[b][32 * c]);
                    f32x2 z[16];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const ulonglong2 k2 = ks[j], v2 = lv[j];
                        f32x2 a = mul2(pk(r[4 * j], r[4 * j + 1]), k2.x), d = mul2(pk(r[4 * j + 2], r[4 * j + 3]), k2.y);
                        if (ASYM) {
                            const ulonglong2 o2 = kl[j];
                            a = fma2(o2.x, qs2, a);
                            d = fma2(o2.y, qs2, d);
                        }
                        z[2 * j] = fma2(a, f2, v2.x);
                        z[2 * j + 1] = fma2(d, f2, v2.y);
                    }
                    if (!plain) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            unsigned u0, u1;
                            unpk(z[j], u0, u1);
                            const int t = tok + 32 * c + 2 * j;
                            if (t < row_lo || t >= row_hi) u0 = 0xff800000u;
                            if (t + 1 < row_lo || t + 1 >= row_hi) u1 = 0xff800000u;
                            z[j] = pk(u0, u1);
                        }
                    }
                    float top = NONE;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        unsigned u0, u1;
                        unpk(z[j], u0, u1);
                        top = max3(__uint_as_float(u0), __uint_as_float(u1), top);
                    }
                    if (__any_sync(0xffffffffu, top > M + MOVE)) {
                        const float mx = fmaxf(M, top), keep = kv_ex2(M - mx);
                        M = mx;
                        const f32x2 keep2 = both(keep);
                        l2 = mul2(l2, keep2);
                        add2v = mul2(add2v, keep2);
                        tmem_st_wait();
                        if (i > 0) {
#pragma unroll 1
                            for (int q = 0; q < 8; ++q) {
                                unsigned o[16];
                                uint4 st[4];
                                tmem_ld16_issue(lanes + O_COL + 16 * q, o);
                                tmem_ld_wait16(o);
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    st[k] = make_uint4(__float_as_uint(__uint_as_float(o[4 * k]) * keep), __float_as_uint(__uint_as_float(o[4 * k + 1]) * keep),
                                                       __float_as_uint(__uint_as_float(o[4 * k + 2]) * keep), __float_as_uint(__uint_as_float(o[4 * k + 3]) * keep));
                                tmem_st16(lanes + O_COL + 16 * q, st);
                            }
                        }
                        const __half2 kh = __float2half2_rn(keep);
#pragma unroll 1
                        for (int q = 0; q < c; ++q) {
                            unsigned o[16];
                            uint4 st[4];
                            tmem_ld16_issue(lanes + 16 * q, o);
                            tmem_ld_wait16(o);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                st[k] = make_uint4(as_u(__hmul2(as_h(o[4 * k]), kh)), as_u(__hmul2(as_h(o[4 * k + 1]), kh)), as_u(__hmul2(as_h(o[4 * k + 2]), kh)),
                                                   as_u(__hmul2(as_h(o[4 * k + 3]), kh)));
                            tmem_st16(lanes + 16 * q, st);
                        }
                    }
                    const ulonglong2* rv = reinterpret_cast<const ulonglong2*>(&S.rv[b][32 * c]);
                    const ulonglong2* vl = reinterpret_cast<const ulonglong2*>(&S.vl[b][32 * c]);
                    const f32x2 base = both(6.f - M);                            // weights are 64 at M
                    uint4 st[4];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const ulonglong2 r2 = rv[j];
                        unsigned h[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            unsigned u0, u1;
                            unpk(add2(z[2 * j + k], base), u0, u1);
                            const float w0 = kv_ex2(__uint_as_float(u0)), w1 = kv_ex2(__uint_as_float(u1));
                            const f32x2 p = mul2(pk(__float_as_uint(w0), __float_as_uint(w1)), k ? r2.y : r2.x);
                            l2 = add2(l2, p);
                            if (ASYM) {
                                const ulonglong2 o2 = vl[j];
                                add2v = fma2(p, k ? o2.y : o2.x, add2v);
                            }
                            h[k] = as_u(__floats2half2_rn(w0, w1));
                        }
                        if (j & 1) { st[j >> 1].z = h[0]; st[j >> 1].w = h[1]; }
                        else { st[j >> 1].x = h[0]; st[j >> 1].y = h[1]; }
                    }
                    tmem_st16(lanes + 16 * c, st);
                }
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(&S.pfull);
            }
            // ---- the rows' sums, by way of shared memory ----
            if (ok && mbar_wait_warp(&S.abort, &S.vfree, (it + n - 1) & 1u, P.status, 77)) {
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    unsigned r[32];
                    tmem_ld32_issue(lanes + O_COL + 32 * c, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4*>(S.k + sum_at(tid, 8 * c + j)) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
                }
            }
            unsigned a, b;
            unpk(l2, a, b);
            S.l[tid] = __uint_as_float(a) + __uint_as_float(b);
            unpk(add2v, a, b);
            S.add[tid] = __uint_as_float(a) + __uint_as_float(b);
            S.m[tid] = M;
            tc_fence_before();
        }
        it += n;
        __syncthreads();
        tc_fence_after();
        const bool starts = piece.starts, ends = piece.ends;
        if (S.abort) break;
        {
            float* part = P.parts + ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * PART;
#pragma unroll 1
            for (int r0 = 0; r0 < ROWS; r0 += 32) {
                const int row = r0 + (tid >> 3), l8 = tid & 7;
                float y[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {                // columns 64 (q >> 1) + 8 l8 + 4 (q & 1) .. hold coordinates 0, 4, 1, 5 (2, 6, 3, 7) of their eight
                    const float4 t = *reinterpret_cast<const float4*>(S.k + sum_at(row, 16 * (q >> 1) + 2 * l8 + (q & 1)));
                    const int at = 8 * (q >> 1) + 2 * (q & 1);
                    y[at] = t.x; y[at + 4] = t.y; y[at + 1] = t.z; y[at + 5] = t.w;
                }
                const float total = S.l[row], extra = S.add[row], m = S.m[row];
                if (starts && ends) {
                    kv_finish(y, l8, 0.f, 6.f, total, extra);
                    if (seg.e.row0 + row < seg.e.rows) {
                        int token, head;
                        kv_row_of(A, seg, row, token, head);
                        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + (seg.e.first + token) * A.out_token + head * A.out_head;
                        if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
                        if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<float4*>(part + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                    if (l8 == 0) {                           // the sums and the totals go by the same M: 64 times their size
                        part[ROWS * 128 + row] = m;
                        part[ROWS * 128 + ROWS + row] = total;
                        part[ROWS * 128 + 2 * ROWS + row] = extra;
                        part[ROWS * 128 + 3 * ROWS + row] = m + 6.f;
                    }
                }
            }
            if (tid == 0 && starts && !ends)
                P.joins[blockIdx.x] = kv_join(P.line, seg, places);
        }
        more = kv_more(P.line, seg, places);
        if (more) kv_next(A, P.line, seg);
        __syncthreads();                                     // shared memory is free for the next segment
    }
    tc_fence_before();
    __syncthreads();
    if (w == 4) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

int blocks_of(const gbs_plan* p) { return p->sm_count * BLOCKS_PER_SM; }

}  // namespace

int64_t gbs_tc_kvattn_workspace(const gbs_plan* p)
{
    return (int64_t)blocks_of(p) * (2 * PART * sizeof(float) + sizeof(KvJoin));
}

int gbs_tc_kvattn_launch(const gbs_plan* p, const gbs_kv_attn& A, void* workspace, cudaStream_t stream)
{
    KvAttnArgs P = {};
    P.a = A;
    P.line.tile_rows = ROWS;
    P.line.unit_log = 7;
    P.line.pad = 3;
    P.line.tiles = (int)(((int64_t)A.max_tokens * A.group + ROWS - 1) / ROWS);
    P.line.by_tiles.set((unsigned)P.line.tiles);
    P.line.entries = A.n_items * P.line.tiles;
    P.line.least = 1;
    const int blocks = blocks_of(p);
    P.joins = static_cast<KvJoin*>(workspace);
    P.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + blocks * sizeof(KvJoin));
    P.status = p->d_status;
    const size_t smem = sizeof(Smem) + 1024;
    const void* f = p->asym ? (const void*)k_tc_kvattn<true> : (const void*)k_tc_kvattn<false>;
    const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    const int rc = gbs_kv_launch(p, p->asym ? k_tc_kvattn<true> : k_tc_kvattn<false>, dim3((unsigned)blocks), THREADS, smem, stream, P);
    if (rc != 0) return rc;
    return gbs_kv_launch(p, k_kv_attn_join<ROWS>, dim3((unsigned)blocks, ROWS / 8), 256, 0, stream, P);
}
