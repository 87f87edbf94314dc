// Attention over the paged KV cache for prompts and chunks of them (gbs_kv_attention, more than 16 query rows of an item and KV head), on
// tcgen05: two tiles of 128 rows (tokens x query heads of a KV head) by 128 cached tokens at a time.
//
// Keys and values enter as fp16 numbers, Delta c (+ lo) times a power of two that 32 tokens have in common, which stays outside:
//     S = Q K^T (fp32 sums),  z = S f 2^Ek,  w = 2^(z + Ev - M + 6),  O += w V,  l += w 2^-Ev.
// f is the row's factor (its power of two, the softmax scale).  With Ev inside the exponent one running maximum M (of z + Ev) serves both the weights'
// range in fp16 and the softmax.  Delta (and the middle of an asymmetric row) is rounded to 11 bits, and the number again, 2^-12 of it each,
// as much as a query coordinate and a weight are.  Exact codes and scales applied to scores and weights instead took three numbers a token from shared
// memory for every row, and 400 us where this takes 318.
//
// Warps 0-3 and 4-7 do the softmax of a tile each, a thread a row; warps 8-11 turn codes into fp16, a thread a token, for both tiles, a
// unit of 128 tokens ahead; warp 12 issues the MMAs.  While one tile's softmax runs, the other's products do.  Scores and weights of a tile share
// 128 columns of tensor memory (fp16 weights overwrite scores that have been read), its sums take 128 more.
// The MMAs take 1024 cycles of a tile, ex2 as many; two tiles of a unit take 5600, most of it the chain of a tile (scores, softmax, weights, second
// product, next scores), which the other tile's overlaps but in part.  The last 2048 of 8048 tokens, 32 query heads over 8 KV heads: 318 us, 740
// TFLOP/s.  Blocks of 128 rows, two on an SM, every warp doing all of it in turn: 433 us.  32 tokens at a time in the softmax: 348.
// 13 warps leave a thread 128 registers, and 74 bytes of one spill.
// Weights reach 2^-30 of the row's largest, below what a bf16 result shows; l is of fp32 weights, which go under when value
// scales that one row sees differ by more than 2^100: the share of the small ones in l is then lost.
#include "gbs_kv_attn.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int TILE = 128, ROWS = 2 * TILE, UNIT = 128;
constexpr int SOFTMAX = ROWS, CODES = UNIT, THREADS = SOFTMAX + CODES + 32;
constexpr int PART = KV_PART<ROWS>;
constexpr float MOVE = 8.f;                          // M moves when a score is so much (log2) above it
constexpr unsigned O_COL = 256, TMEM_COLS = 512;     // scores of tile t from column 128 t on, sums from O_COL + 128 t on

struct Smem {
    unsigned char q[2][TILE * 256];                  // fp16, K-major, two blocks of 64 coordinates, 128-byte swizzle
    unsigned char k[2][UNIT * 256];                  // the same, unit i in [i & 1]; at a segment's end k holds the first tile's sums in fp32, v the second's
    unsigned char v[2][UNIT * 256];                  // N-major for the second product: the same bytes
    float4 part[4][UNIT / 32];                       // of 32 tokens of unit i, in [i & 3]: 2^Ek, Ev, 2^-Ev, and (as bits) which tokens are there
    float factor[ROWS];
    int lo[ROWS], hi[ROWS];                          // tokens that a row sees
    float m[ROWS], l[ROWS];
    unsigned long long kfull[2], kfree[2], vfull[2], vfree[2], sfull[2], pfull[2], ofull, drain;
    KvSeg seg[2];                                    // of segment i in [i & 1]: registers are scarce, and a spilled one is fetched from L2
    long long share[THREADS / 32];
    unsigned tmem;
    int abort;
};
static_assert(sizeof(Smem) + 1024 <= 227 * 1024, "one block of an SM");

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 both(float x) { return pk(__float_as_uint(x), __float_as_uint(x)); }
template <int N>
struct Is { static constexpr int value = N; };
// a number that is the same in all lanes, as the compiler then knows
__device__ __forceinline__ unsigned uniform(unsigned x) { return __shfl_sync(0xffffffffu, x, 0); }
// the block's warps meet, wherever in the code they are
__device__ __forceinline__ void meet_all() { asm volatile("bar.sync 0, %0;" ::"n"(THREADS) : "memory"); }
// The same, and whether any of their threads says so: all of them leave, or none.  (The flag of the waits may be raised between two reads of it.)
__device__ __forceinline__ bool meet_any(bool x)
{
    int any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((int)x), "n"(THREADS) : "memory");
    return any != 0;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st32(unsigned taddr, const unsigned r[32])
{
    tmem_st16(taddr, reinterpret_cast<const uint4*>(r));
    tmem_st16(taddr + 16, reinterpret_cast<const uint4*>(r + 16));
}

// byte of a 16-byte piece (8 coordinates) of a row in a tile
__device__ __forceinline__ unsigned piece_at(int row, int piece)
{
    return (unsigned)(piece >> 3) * (128 * 128) + (unsigned)(row >> 3) * 1024 + (unsigned)(row & 7) * 128 + (unsigned)(((piece & 7) ^ (row & 7)) << 4);
}
// byte of a 16-byte piece (4 coordinates) of a row of sums
__device__ __forceinline__ unsigned sum_at(int row, int piece) { return (unsigned)row * 512 + (unsigned)((piece ^ (row & 31)) << 4); }

// A row's codes (64 bytes) to fp16, c scale + middle with c in -8 .. 7.  A word's 8 coordinates stand in the order 0, 4, 1, 5, 2, 6, 3, 7, in the
// queries as well; the results' columns are put back at the end.
template <bool ASYM>
__device__ __forceinline__ void store_codes(unsigned char* tile, int row, const uint4 codes[4], __half2 scale, __half2 middle)
{
    // nibbles (i, i + 4) in the mantissas of 1024 (of 64, times 16), a symmetric code as c ^ 8 = c + 8
    constexpr unsigned LOW = ASYM ? 0x64006400u : 0x64086408u, HIGH = ASYM ? 0x64006400u : 0x64806480u;
    const __half2 off = __float2half2_rn(1032.f), off16 = __float2half2_rn(-72.f), by = __float2half2_rn(0.0625f);
    const unsigned first = smem_u32(tile) + piece_at(row, 0);        // a tile starts on 1024 bytes: the piece's number is exclusive-or'ed in
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint4 q = codes[i >> 2];
        const unsigned w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w, w8 = w >> 8;
        __half2 c[4] = {__hsub2(as_h(kv_and_xor(w, 0x000f000fu, LOW)), off), __hfma2(as_h(kv_and_xor(w, 0x00f000f0u, HIGH)), by, off16),
                        __hsub2(as_h(kv_and_xor(w8, 0x000f000fu, LOW)), off), __hfma2(as_h(kv_and_xor(w8, 0x00f000f0u, HIGH)), by, off16)};
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = ASYM ? __hfma2(c[k], scale, middle) : __hmul2(c[k], scale);
        st_shared_v4((first ^ (unsigned)((i & 7) << 4)) + (i >> 3) * (128 * 128), make_uint4(as_u(c[0]), as_u(c[1]), as_u(c[2]), as_u(c[3])));
    }
}
// The power of two of 32 tokens whose largest number is `most`: it takes that just below 2^8, far from fp16's smallest ones.  0: none.
__device__ __forceinline__ int power_of(float most) { return max((int)(__float_as_uint(most) >> 23) - 134, -100); }
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ void load_codes(uint4 c[4], const unsigned char* from)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = reinterpret_cast<const uint4*>(from)[i];
}

// What a thread's row has added up, and the weights of the unit's first 32 `weights` tokens, times `keep`; rare.
__device__ __forceinline__ void shrink(unsigned scores, unsigned sums, float keep, bool have, int weights)
{
    tmem_st_wait();
    if (have) {
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
            unsigned o[32];
            tmem_ld32_issue(sums + 32 * q, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * keep);
            tmem_st32(sums + 32 * q, o);
        }
    }
    const __half2 h = __float2half2_rn(keep);
#pragma unroll 1
    for (int q = 0; q < weights; ++q) {
        unsigned o[16], unused[16] = {};
        tmem_ld16_issue(scores + 16 * q, o);
        tmem_ld_wait16x2(o, unused);
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = as_u(__hmul2(as_h(o[k]), h));
        tmem_st16(scores + 16 * q, reinterpret_cast<const uint4*>(o));
    }
}

template <bool ASYM, bool TEST>
__global__ __launch_bounds__(THREADS, 1) void k_tc_kvattn(const __grid_constant__ KvAttnArgs P)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = warp_index();
    if (tid == 0) {
        S.abort = 0;
        for (int b = 0; b < 2; ++b) {
            mbar_init(&S.kfull[b], CODES / 32);
            mbar_init(&S.vfull[b], CODES / 32);
            mbar_init(&S.kfree[b], 1);
            mbar_init(&S.vfree[b], 1);
            mbar_init(&S.sfull[b], 2);                       // the MMAs, and the thread that has seen the per-token numbers
            mbar_init(&S.pfull[b], TILE / 32);
        }
        mbar_init(&S.ofull, 1);
        mbar_init(&S.drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == 12) tmem_alloc(&S.tmem, TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = S.tmem;
    kv_wait_before();
    kv_let_next();

    const int places = kv_share<THREADS>(A, P.line, &S.seg[0], S.share);
    if (tid == 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};

    const int ps_log = A.c.page_log, ps = 1 << ps_log;
    unsigned it = 0, round = 0, phase_b = 0;                 // units, segments and the second tile's units so far, by which the barriers' phases go
    for (bool more = places > 0; more; ++round) {
        const KvSeg& seg = S.seg[round & 1];
        const KvPiece piece = kv_piece(P.line, seg, places);
        const int n = piece.n, tok0 = (seg.e.lo / UNIT + piece.skip) * UNIT;
        if (n <= 0) break;                                   // the block's last places are in front of a segment's units
        const bool two = seg.e.row0 + TILE < seg.e.rows;     // the second tile has rows
        bool ok = true;

        if (w < SOFTMAX / 32) {
            // ---- query rows: eight lanes a row, 32 rows at a time ----
#pragma unroll 1
            for (int q0 = 0; q0 < (two ? ROWS : TILE); q0 += 128) {
                const int l8 = tid & 7;
                uint4 raw[4][2];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = q0 + 32 * r + (tid >> 3);
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
                    const int row = q0 + 32 * r + (tid >> 3);
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
                    const float turned = copysignf(down, A.scale);       // f > 0: a masked score, and the largest one, stay what they are
                    __half h[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) h[i] = __float2half_rn(y[i] * turned);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const __half* g = h + 8 * half;
                        *reinterpret_cast<uint4*>(S.q[row >> 7] + piece_at(row & 127, 8 * half + l8)) =
                            make_uint4(as_u(__halves2half2(g[0], g[4])), as_u(__halves2half2(g[1], g[5])), as_u(__halves2half2(g[2], g[6])), as_u(__halves2half2(g[3], g[7])));
                    }
                    if (l8 == 0) {
                        S.factor[row] = up * (fabsf(A.scale) * (KV_NORM * 1.4426950408889634f));
                        const int token = A.by_group(min(seg.e.row0 + row, seg.e.rows - 1));
                        S.lo[row] = kv_row_lo(A, seg.e, token);
                        S.hi[row] = seg.e.row0 + row < seg.e.rows ? kv_row_hi(A, seg.e, token) : 0;
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            meet_all();

            const int t = w >> 2, row = tid;                 // this thread's tile and row
            const unsigned scores = tmem + ((unsigned)(32 * (w & 3)) << 16) + 128 * t, sums = scores + O_COL;
            const float f = S.factor[row];
            const int see_lo = S.lo[row], see_hi = S.hi[row];
            // tokens that every row of the tile sees need no mask
            const int first = seg.e.row0 + TILE * t;
            const int all_lo = kv_row_lo(A, seg.e, A.by_group(min(seg.e.rows, first + TILE) - 1)), all_hi = kv_row_hi(A, seg.e, A.by_group(first));
            float M = NONE;
            f32x2 l = both(0.f);                             // of even and odd tokens
            for (int i = 0; i < n && ok && (t == 0 || two); ++i) {
                const unsigned now = it + i;
                const int nb = now & 3, tok = tok0 + i * UNIT;
                const bool plain = tok >= all_lo && tok + UNIT <= all_hi;
                if (!(ok = !kv_lost<TEST>(P, &S.abort, 76, round) && mbar_wait_warp(&S.abort, &S.sfull[t], (t == 0 ? now : phase_b + i) & 1u, P.status, 76))) break;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {                // 64 tokens at a time
                    unsigned x[2][32];
                    tmem_ld32_issue(scores + 64 * c, x[0]);
                    tmem_ld32_issue(scores + 64 * c + 32, x[1]);
                    const float4 part[2] = {S.part[nb][2 * c], S.part[nb][2 * c + 1]};
                    float fc[2], most[2];
                    tmem_ld_wait(x[0]);
                    tmem_ld_wait(x[1]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        fc[h] = fmaxf(f * part[h].x, 7.5e-37f);          // not 0, for a masked score's sake
                        const unsigned there = __float_as_uint(part[h].w);
                        if (!plain || there != 0xffffffffu) {
                            const int lo = see_lo - tok - 64 * c - 32 * h, hi = see_hi - tok - 64 * c - 32 * h;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < lo || j >= hi || !(there >> j & 1)) x[h][j] = 0xff800000u;
                        }
                        float top[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) top[j] = fmaxf(__uint_as_float(x[h][8 * j]), __uint_as_float(x[h][8 * j + 1]));
#pragma unroll
                        for (int k = 2; k < 8; k += 2)
#pragma unroll
                            for (int j = 0; j < 4; ++j) top[j] = max3(__uint_as_float(x[h][8 * j + k]), __uint_as_float(x[h][8 * j + k + 1]), top[j]);
                        most[h] = fmaxf(max3(top[0], top[1], top[2]), top[3]) * fc[h] + part[h].y;
                    }
                    most[0] = fmaxf(most[0], most[1]);
                    if (__any_sync(0xffffffffu, most[0] > M + MOVE)) {
                        // rare: what has been added up by the old maximum shrinks
                        const float now_M = fmaxf(most[0], M), keep = kv_ex2(M - now_M);
                        M = now_M;
                        l = mul2(l, both(keep));
                        shrink(scores, sums, keep, i > 0, 2 * c);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x2 f2 = both(fc[h]), base = both(6.f - M + part[h].y);      // weights are 64 at M
                        unsigned p[16];
                        f32x2 l2[2] = {both(0.f), both(0.f)};
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            unsigned u0, u1;
                            unpk(fma2(pk(x[h][2 * j], x[h][2 * j + 1]), f2, base), u0, u1);
                            const float w0 = kv_ex2(__uint_as_float(u0)), w1 = kv_ex2(__uint_as_float(u1));
                            l2[j & 1] = add2(l2[j & 1], pk(__float_as_uint(w0), __float_as_uint(w1)));
                            p[j] = as_u(__floats2half2_rn(w0, w1));
                        }
                        l = fma2(add2(l2[0], l2[1]), both(part[h].z), l);
                        tmem_st16(scores + 32 * c + 16 * h, reinterpret_cast<const uint4*>(p));
                    }
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.pfull[t]);
            }
            // ---- the rows' sums, by way of shared memory ----
            if (ok && (t == 0 || two) && (ok = !kv_lost<TEST>(P, &S.abort, 77, round) && mbar_wait_warp(&S.abort, &S.ofull, round & 1u, P.status, 77))) {
                tc_fence_after();
                unsigned char* to = t == 0 ? S.k[0] : S.v[0];
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    unsigned r[32];
                    tmem_ld32_issue(sums + 32 * c, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4*>(to + sum_at(row & 127, 8 * c + j)) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
                }
                unsigned u0, u1;
                unpk(l, u0, u1);
                S.l[row] = __uint_as_float(u0) + __uint_as_float(u1);
                S.m[row] = M;
            }
            tc_fence_before();
            if (meet_any(!ok)) break;
            tc_fence_after();
            float* parts = P.parts + ((long long)blockIdx.x * 2 + (piece.starts ? 1 : 0)) * PART;
#pragma unroll 1
            for (int q0 = 0; q0 < (two ? ROWS : TILE); q0 += 32) {
                const int row = q0 + (tid >> 3), l8 = tid & 7;
                const unsigned char* from = row < TILE ? S.k[0] : S.v[0];
                float y[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {                // columns 64 (q >> 1) + 8 l8 + 4 (q & 1) .. hold coordinates 0, 4, 1, 5 (2, 6, 3, 7) of their eight
                    const float4 x = *reinterpret_cast<const float4*>(from + sum_at(row & 127, 16 * (q >> 1) + 2 * l8 + (q & 1)));
                    const int at = 8 * (q >> 1) + 2 * (q & 1);
                    y[at] = x.x; y[at + 4] = x.y; y[at + 1] = x.z; y[at + 5] = x.w;
                }
                const float total = S.l[row], m = S.m[row];
                if (piece.starts && piece.ends) {
                    kv_finish(y, l8, 0.f, 6.f, total, 0.f);
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
                        *reinterpret_cast<float4*>(parts + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                    if (l8 == 0) {                           // the sums and the totals go by the same M: 64 times their size
                        parts[ROWS * 128 + row] = m;
                        parts[ROWS * 128 + ROWS + row] = total;
                        parts[ROWS * 128 + 2 * ROWS + row] = 0.f;
                        parts[ROWS * 128 + 3 * ROWS + row] = m + 6.f;
                    }
                }
            }
            if (tid == 0 && piece.starts && !piece.ends) P.joins[blockIdx.x] = kv_join(P.line, seg, places);
            if (t == 1 && two) phase_b += n;
        } else if (w < 12) {
            // ---- codes: keys and values of a unit, and its per-token numbers ----
            const int me = tid - SOFTMAX;                    // this thread's token of a unit
            const int slot = me & (ps - 1), k_at = slot * KV_ROW, v_at = k_at + ps * KV_ROW;
            const int* pages = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            const auto page_of = [&](int tok) { return tok < seg.e.hi ? pages[tok >> ps_log] : -1; };
            // where a token's block is; some block of the pool, whose codes will weigh nothing, where it is not there to be seen
            const auto find = [&](int tok, int page, bool& there) {
                there = tok >= seg.e.lo && tok < seg.e.hi && (unsigned)page < (unsigned)A.c.n_pages;
                return static_cast<const unsigned char*>(kv_block(A.c, there ? page : 0, seg.head));
            };
            bool there;
            const unsigned char* block = find(tok0 + me, page_of(tok0 + me), there);
            int page = page_of(tok0 + UNIT + me);
            uint4 k[4], v[4];
            float ks, kl, vs, vl;
            const auto load = [&] {
                load_codes(k, block + k_at);
                const float* sc = reinterpret_cast<const float*>(block + 2 * ps * KV_ROW);
                kl = vl = 0.f;
                if (ASYM) {
                    const float2 a = reinterpret_cast<const float2*>(sc)[slot], b = reinterpret_cast<const float2*>(sc)[ps + slot];
                    ks = a.x; kl = a.y; vs = b.x; vl = b.y;
                } else {
                    ks = sc[slot];
                    vs = sc[ps + slot];
                }
                load_codes(v, block + v_at);
            };
            load();
            int ev = -60;                                    // far below any values'
            meet_all();                                 // the segment's queries are there, and shared memory is free
            for (int i = 0; i < n; ++i) {
                const unsigned now = it + i, use = now >> 1;
                const int b = now & 1, nb = now & 3;
                if (now > 1 && !(ok = !kv_lost<TEST>(P, &S.abort, 74, round) && mbar_wait_warp(&S.abort, &S.kfree[b], (use + 1) & 1u, P.status, 74))) break;
                // tokens that are not there become 0, those whose scales are no numbers NaN keys: the scores of rows that see them are none
                const bool wrong = !(fabsf(ks) + fabsf(vs) + fabsf(kl) + fabsf(vl) < INFINITY);
                if (!there || wrong) ks = kl = vs = vl = 0.f;
                const float km = ASYM ? fmaf(8.f, ks, kl) : 0.f, vm = ASYM ? fmaf(8.f, vs, vl) : 0.f;
                const float most_k = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fabsf(ks), fabsf(km)))));
                const float most_v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fabsf(vs), fabsf(vm)))));
                const int ek = power_of(most_k);
                if (most_v > 0.f) ev = power_of(most_v);             // where all are 0, any power will do, but for M
                const float up = two_to(-ek), up_v = two_to(-ev);
                const unsigned which = __ballot_sync(0xffffffffu, there);
                if (lane == 0) S.part[nb][w - 8] = make_float4(two_to(ek), (float)ev, two_to(-ev), __uint_as_float(which));
                store_codes<ASYM>(S.k[b], me, k, there && wrong ? as_h(0x7fff7fffu) : __float2half2_rn(ks * up), __float2half2_rn(km * up));
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.kfull[b]);
                if (now > 1 && !(ok = !kv_lost<TEST>(P, &S.abort, 75, round) && mbar_wait_warp(&S.abort, &S.vfree[b], (use + 1) & 1u, P.status, 75))) break;
                store_codes<ASYM>(S.v[b], me, v, __float2half2_rn(vs * up_v), __float2half2_rn(vm * up_v));
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.vfull[b]);
                if (i + 1 < n) {
                    const int next = tok0 + (i + 1) * UNIT + me;
                    block = find(next, page, there);
                    page = page_of(next + UNIT);
                    load();
                }
            }
            if (meet_any(!ok)) break;                   // the sums are there
        } else {
            // ---- MMAs: weights times values of a unit, then the next one's scores, for one tile and the other in turn ----
            // Everything that an MMA takes is made uniform, and what changes between them is known when this is compiled: see umma_f16.
            constexpr unsigned ID_S = (1u << 4) | ((unsigned)(UNIT >> 3) << 17) | ((unsigned)(TILE >> 4) << 24);             // fp16, both K-major
            constexpr unsigned ID_O = ID_S | (1u << 16);                                                                    // B N-major
            constexpr unsigned TILE_STEP = (TILE * 256) >> 4;
            const unsigned long long qd = smem_desc(smem_u32(S.q[0]), 16, 1024, 2), kd = smem_desc(smem_u32(S.k[0]), 16, 1024, 2),
                                     vd = smem_desc(smem_u32(S.v[0]), 128 * 128, 1024, 2);
            const unsigned q_lo = (unsigned)qd, k_lo = (unsigned)kd, v_lo = (unsigned)vd, hi = (unsigned)(qd >> 32);          // the same in all three
            const unsigned at = uniform(tmem), at0 = uniform(it), at0_b = uniform(phase_b);
            const int units = (int)uniform((unsigned)n), tiles = uniform(two ? 2u : 1u);
            const auto scores = [&](auto tile, unsigned b) {
                constexpr int t = decltype(tile)::value;
                unsigned a_lo = q_lo + t * TILE_STEP, b_lo = k_lo + b * TILE_STEP;
                umma_f16_words<false>(at + 128 * t, a_lo, hi, b_lo, hi, ID_S);
#pragma unroll
                for (int k = 1; k < 8; ++k) {                // sixteen coordinates: 32 bytes, four of them in a block of 64
                    const unsigned step = (k & 3) ? 2u : (unsigned)((TILE * 128 - 96) >> 4);
                    a_lo += step;
                    b_lo += step;
                    umma_f16_words<true>(at + 128 * t, a_lo, hi, b_lo, hi, ID_S);
                }
                umma_commit(&S.sfull[t]);
                if (lane == 0) mbar_arrive(&S.sfull[t]);
            };
            const auto values = [&](auto tile, auto adds, unsigned b) {
                constexpr int t = decltype(tile)::value;
                unsigned b_lo = v_lo + b * TILE_STEP;
                umma_f16_ts(at + O_COL + 128 * t, at + 128 * t, (unsigned long long)hi << 32 | b_lo, ID_O, decltype(adds)::value);
#pragma unroll
                for (int k = 1; k < 8; ++k) {                // sixteen tokens: two groups of eight rows
                    b_lo += 2048 >> 4;
                    umma_f16_ts(at + O_COL + 128 * t, at + 128 * t + 8 * k, (unsigned long long)hi << 32 | b_lo, ID_O, 1);
                }
            };
            constexpr Is<0> A_TILE; constexpr Is<1> B_TILE;
            meet_all();
            // the first scores, and so on: one function for a tile's part of a step
            const auto step = [&](auto tile, auto adds, int i) {
                constexpr int t = decltype(tile)::value;
                const unsigned now = at0 + i, next = now + 1;
                if (i >= 0) {
                    if (t == 0 && (kv_lost<TEST>(P, &S.abort, 72, round) || !mbar_wait_warp(&S.abort, &S.vfull[now & 1], (now >> 1) & 1u, P.status, 72))) return false;
                    if (kv_lost<TEST>(P, &S.abort, 73, round) || !mbar_wait_warp(&S.abort, &S.pfull[t], (t == 0 ? now : at0_b + i) & 1u, P.status, 73)) return false;
                    tc_fence_after();
                    values(tile, adds, now & 1);
                    if (t + 1 == tiles) umma_commit(&S.vfree[now & 1]);
                }
                if (i + 1 < units) {
                    if (t == 0) {
                        if (kv_lost<TEST>(P, &S.abort, 71, round) || !mbar_wait_warp(&S.abort, &S.kfull[next & 1], (next >> 1) & 1u, P.status, 71)) return false;
                        tc_fence_after();
                    }
                    scores(tile, next & 1);
                    if (t + 1 == tiles) umma_commit(&S.kfree[next & 1]);
                }
                return true;
            };
            const auto unit = [&](auto adds, int i) { return step(A_TILE, adds, i) && (tiles == 1 || step(B_TILE, adds, i)); };
            ok = unit(Is<0>{}, -1) && unit(Is<0>{}, 0);
            for (int i = 1; i < units && ok; ++i) ok = unit(Is<1>{}, i);
            if (ok) umma_commit(&S.ofull);
            else {                                           // what is under way is given time to end
                umma_commit(&S.drain);
                drain_copies(&S.drain, 1, 1);
            }
            if (two) phase_b += n;
            if (lane == 0 && kv_more(P.line, seg, places)) {
                KvSeg next = seg;
                kv_next(A, P.line, next);
                S.seg[(round + 1) & 1] = next;
            }
            if (meet_any(!ok)) {
                if (ok) drain_copies(&S.ofull, 1, (int)round + 1);       // the products are given time to end, as above
                break;
            }
        }
        it += n;
        more = kv_more(P.line, seg, places);
    }
    tc_fence_before();
    __syncthreads();
    if (w == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

int blocks_of(const gbs_plan* p) { return p->sm_count; }

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
    P.line.pad = 5;                                  // queries and results take as long as five units (2: 134 us for six prompts of up to 1700 tokens, 3: 117, 5: 102, 9: 106)
    P.line.tiles = (int)(((int64_t)A.max_tokens * A.group + ROWS - 1) / ROWS);
    P.line.by_tiles.set((unsigned)P.line.tiles);
    P.line.entries = A.n_items * P.line.tiles;
    P.line.least = 1;
    const int blocks = blocks_of(p);
    P.joins = static_cast<KvJoin*>(workspace);
    P.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + blocks * sizeof(KvJoin));
    P.status = p->d_status;
    const size_t smem = sizeof(Smem) + 1024;
    const auto f = A.lost_code ? (p->asym ? k_tc_kvattn<true, true> : k_tc_kvattn<false, true>)
                               : (p->asym ? k_tc_kvattn<true, false> : k_tc_kvattn<false, false>);
    const cudaError_t e = cudaFuncSetAttribute((const void*)f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    const int rc = gbs_kv_launch(p, f, dim3((unsigned)blocks), THREADS, smem, stream, P);
    if (rc != 0) return rc;
    return gbs_kv_launch(p, k_kv_attn_join<ROWS>, dim3((unsigned)blocks, ROWS / 8), 256, 0, stream, P);
}
