// Attention over the paged KV cache for few query rows (gbs_kv_attention: decoding).
//
// With khat = Delta c (+ lo) in the rotated basis, scores are Delta_k (H q . c) (+ lo sum H q) and the result is H sum_j (p_j Delta_v) c_j
// (+ sum_j p_j lo_j): the codes go into the matrix unit as they are, exactly, and the rotation is applied to eight query rows and
// eight results instead of to every cached row.
//
// What bounds it is the cache, 136 or 144 bytes a token and KV head, read once.  The matrix unit takes 16 rows at a time; there are at
// most eight here, so each is given as a sum of two, q = hi + lo 2^-11 in fp16 and p Delta_v = hi + lo in bf16: 22 and 16 bits at no cost, and
// both halves of a row land in the same thread.  Layouts are chosen so that codes go from shared memory to the operand registers
// without being moved between threads: the order of the 128 coordinates of a score, of a group's 8 tokens and of the 128 columns of the
// result is free, as long as both operands have the same.  A nibble becomes a number by or-ing it into the low mantissa bits of 1024
// (fp16) or 128 (bf16) and subtracting that, exactly.
//
// A warp works alone: it fetches units of 32 tokens (bulk copies into a ring of its own), keeps sums for its tokens in registers, and
// meets the block's other warps where a segment ends.  The running maximum is moved only when a score exceeds it by 2^8.
#include <cuda_fp16.h>

#include "gbs_kv_sched.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int ROWS = 8, UNIT = 32;
constexpr int WARPS = 6, THREADS = 32 * WARPS, STAGES = 3;
constexpr int PART = ROWS * 128 + 3 * ROWS;          // floats of a partial result: sums, maximum, total, sum of p lo
constexpr int BLOCKS_PER_SM = 2;
constexpr float MOVE = 8.f;                          // the maximum moves when a score is so much (log2) above it

template <bool ASYM>
struct Stage {
    static constexpr int SCALE = UNIT * (ASYM ? 8 : 4);
    unsigned char k[UNIT * KV_ROW], v[UNIT * KV_ROW];
    unsigned char ks[SCALE], vs[SCALE];
};

template <bool ASYM>
struct Smem {
    Stage<ASYM> ring[WARPS][STAGES];
    float part[WARPS][ROWS * 128];                   // 16-byte pieces in the order piece ^ (lane & 7) of each thread's eight
    float m[WARPS][ROWS], l[WARPS][ROWS], add[WARPS][ROWS];
    __half qh[ROWS][128], ql[ROWS][128];             // coordinates in the order of the operand, see place()
    float factor[ROWS], qsum[ROWS];
    unsigned long long full[WARPS][STAGES];
    unsigned valid[WARPS][STAGES];                   // bit h: tokens 16 h .. of the unit have a page
    KvSeg ahead[WARPS];                              // the segment of the next unit to fetch
    long long share[WARPS + 3];
    int abort;
};

struct Args {
    gbs_kv_attn a;
    KvLine line;
    float* parts;                                    // [blocks][2][PART]
    KvJoin* joins;                                   // [blocks]
    int* status;
};

__device__ __forceinline__ void mma_f16(float c[4], const unsigned a[4], unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float c[4], const unsigned a[4], unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ unsigned as_u(__half2 x) { return *reinterpret_cast<unsigned*>(&x); }
__device__ __forceinline__ unsigned as_u(__nv_bfloat162 x) { return *reinterpret_cast<unsigned*>(&x); }
__device__ __forceinline__ __half2 as_h(unsigned x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ __nv_bfloat162 as_b(unsigned x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Eight codes of a word -> pairs (0, 4), (1, 5), (2, 6), (3, 7) in fp16.  A symmetric code c is kept as c ^ 8 = c + 8 of four bits.
template <bool ASYM>
__device__ __forceinline__ void codes_f16(unsigned w, unsigned out[4])
{
    constexpr unsigned LOW = ASYM ? 0x64006400u : 0x64086408u, HIGH = ASYM ? 0x64006400u : 0x64806480u;
    const __half2 off = __float2half2_rn(ASYM ? 1024.f : 1032.f), off16 = __float2half2_rn(ASYM ? -64.f : -72.f), by = __float2half2_rn(0.0625f);
    const unsigned w8 = w >> 8;
    out[0] = as_u(__hsub2(as_h((w & 0x000f000fu) ^ LOW), off));
    out[1] = as_u(__hfma2(as_h((w & 0x00f000f0u) ^ HIGH), by, off16));
    out[2] = as_u(__hsub2(as_h((w8 & 0x000f000fu) ^ LOW), off));
    out[3] = as_u(__hfma2(as_h((w8 & 0x00f000f0u) ^ HIGH), by, off16));
}
// Four codes of token a (low half) and of token b (high half) -> four pairs (a_i, b_i) in bf16.
template <bool ASYM>
__device__ __forceinline__ void codes_bf16(unsigned w, unsigned out[4])
{
    constexpr unsigned LOW = ASYM ? 0x43004300u : 0x43084308u;
    const __nv_bfloat162 off = __float2bfloat162_rn(ASYM ? 128.f : 136.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = as_u(__hsub2(as_b(((w >> (4 * i)) & 0x000f000fu) ^ LOW), off));
}

// where coordinate 32 t + 8 w + n stands in a query row: operand register (w, n & 3) of thread t holds n and n + 4
__device__ __forceinline__ void store_row(__half* row, int l8, const __half h[16])
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const __half* x = h + 8 * half;
        uint4 u;
        u.x = as_u(__halves2half2(x[0], x[4]));
        u.y = as_u(__halves2half2(x[1], x[5]));
        u.z = as_u(__halves2half2(x[2], x[6]));
        u.w = as_u(__halves2half2(x[3], x[7]));
        *reinterpret_cast<uint4*>(row + 64 * half + 8 * l8) = u;
    }
}

// row of a tile -> token of the item and query head
__device__ __forceinline__ void row_of(const gbs_kv_attn& A, const KvSeg& s, int row, int& token, int& head)
{
    const int r = s.e.row0 + row;
    token = r / A.group;
    head = s.head * A.group + (r - token * A.group);
}

template <bool ASYM>
__global__ __launch_bounds__(THREADS, BLOCKS_PER_SM) void k_kv_attn_few(const __grid_constant__ Args P)
{
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Smem<ASYM>& S = *reinterpret_cast<Smem<ASYM>*>(smem_raw);
    const gbs_kv_attn& A = P.a;
    const int lane = threadIdx.x & 31, w = warp_index(), g = lane >> 2, t = lane & 3;
    if (threadIdx.x == 0) S.abort = 0;
    if (lane < STAGES) mbar_init(&S.full[w][lane], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    kv_wait_before();
    kv_let_next();

    KvSeg seg;
    const int units = kv_share<THREADS>(A, P.line, seg, S.share);
    if (threadIdx.x == 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};
    if (units == 0) return;

    // ---- fetching: units w, w + WARPS, .. of the block's line ----
    const int ps_log = A.c.page_log, T = min(UNIT, 1 << ps_log);
    const int pieces = T == UNIT ? 4 : 8, half = lane >> 2, piece = lane & 3;
    const unsigned piece_bytes = piece < 2 ? T * KV_ROW : T * (ASYM ? 8 : 4);
    const int in_block = piece < 2 ? piece * (KV_ROW << ps_log) : (2 * KV_ROW << ps_log) + (piece - 2) * ((ASYM ? 8 : 4) << ps_log);
    const int in_slot = piece < 2 ? KV_ROW : (ASYM ? 8 : 4);
    const int in_stage = (piece < 2 ? piece * UNIT * KV_ROW : 2 * UNIT * KV_ROW + (piece - 2) * Stage<ASYM>::SCALE) + half * (int)piece_bytes;
    int fetch = w, fetch_page = -1, fetch_tok = 0, fetched = 0;             // the next unit, this lane's page and token of it
    // (a lane below `pieces` copies one piece)
    auto look = [&]() {
        KvSeg* a = &S.ahead[w];
        if (fetch >= units) return;
        if (fetch >= a->at + a->e.units) {
            KvSeg s = *a;
            while (fetch >= s.at + s.e.units) kv_next(A, s, P.line.entries, P.line.tiles, ROWS, UNIT);
            __syncwarp();
            if (lane == 0) *a = s;
            __syncwarp();
        }
        fetch_tok = (a->e.lo / UNIT + fetch - a->at) * UNIT + half * 16;
        fetch_page = -1;
        if (lane < pieces && fetch_tok < a->e.hi) fetch_page = kv_page(A.c, a->e.seq, fetch_tok);
    };
    auto issue = [&]() {
        if (fetch >= units) return;
        const int st = fetched % STAGES;
        const bool ok = fetch_page >= 0;
        const unsigned who = __ballot_sync(0xffffffffu, ok);
        const unsigned valid = T == UNIT ? ((who & 1) ? 3u : 0u) : (who & 1) | ((who >> 4) & 1) << 1;
        const int head = S.ahead[w].head;
        if (lane == 0) {
            S.valid[w][st] = valid;
            mbar_arrive_expect_tx(&S.full[w][st], (unsigned)(((who & 1) + ((who >> 4) & 1)) * T * (2 * KV_ROW + (ASYM ? 16 : 8))));
        }
        __syncwarp();
        if (ok)
            bulk_load(reinterpret_cast<unsigned char*>(&S.ring[w][st]) + in_stage,
                      kv_block(A.c, fetch_page, head) + in_block + (fetch_tok & ((1 << ps_log) - 1)) * in_slot, piece_bytes, &S.full[w][st]);
        ++fetched;
        fetch += WARPS;
        look();
    };
    if (lane == 0) S.ahead[w] = seg;
    __syncwarp();
    look();
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) issue();

    // ---- the segments ----
    int mine = w, done = 0;                              // this warp's next unit of the line, units it has worked on
    bool dead = false;
    for (;;) {
        // query rows: four of them per warp, rotated, halved
        if (w < 2) {
            const int row = 4 * w + (lane >> 3), l8 = lane & 7;
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (seg.e.row0 + row < seg.e.rows) {
                int token, head;
                row_of(A, seg, row, token, head);
                const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(A.q) + (seg.e.first + token) * A.q_token + head * A.q_head;
                if (8 * l8 < A.d) a = *reinterpret_cast<const uint4*>(x + 8 * l8);
                if (64 + 8 * l8 < A.d) b = *reinterpret_cast<const uint4*>(x + 64 + 8 * l8);
            }
            float y[16];
            kv_unpack_bf16(a, y);
            kv_unpack_bf16(b, y + 8);
            kv_hadamard(y, l8);
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(y[i]));
#pragma unroll
            for (int h = 1; h < 8; h <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, h));
            const int e = min(max((int)(__float_as_uint(m) >> 23), 1), 252);
            const float down = __uint_as_float((unsigned)(253 - e) << 23), up = __uint_as_float((unsigned)(e + 1) << 23);     // 2^(126-e), its inverse
            __half hi[16], lo[16];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = y[i] * down;
                hi[i] = __float2half_rn(v);
                lo[i] = __float2half_rn((v - __half2float(hi[i])) * 2048.f);
                sum += __half2float(hi[i]) + __half2float(lo[i]) * (1.f / 2048.f);
            }
#pragma unroll
            for (int h = 1; h < 8; h <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, h);
            store_row(S.qh[row], l8, hi);
            store_row(S.ql[row], l8, lo);
            if (l8 == 0) {
                S.factor[row] = up * (A.scale * (KV_NORM * 1.4426950408889634f));
                S.qsum[row] = sum;
            }
        }
        __syncthreads();
        unsigned qa[8][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 h = *reinterpret_cast<const uint4*>(&S.qh[g][32 * t + 8 * i]), l = *reinterpret_cast<const uint4*>(&S.ql[g][32 * t + 8 * i]);
            qa[2 * i][0] = h.x; qa[2 * i][2] = h.y; qa[2 * i + 1][0] = h.z; qa[2 * i + 1][2] = h.w;
            qa[2 * i][1] = l.x; qa[2 * i][3] = l.y; qa[2 * i + 1][1] = l.z; qa[2 * i + 1][3] = l.w;
        }
        const float factor = S.factor[g], qsum = S.qsum[g] * factor;
        const int my_token = min(seg.e.row0 + g, seg.e.rows - 1) / A.group;
        const int row_lo = kv_row_lo(A, seg.e, my_token), row_hi = kv_row_hi(A, seg.e, my_token);
        // tokens that all rows of the tile see need no mask
        const int all_lo = kv_row_lo(A, seg.e, (min(seg.e.rows, seg.e.row0 + ROWS) - 1) / A.group), all_hi = kv_row_hi(A, seg.e, seg.e.row0 / A.group);

        float o[16][4];
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        float m = -INFINITY, l = 0.f, add = 0.f;
        const unsigned order = (t & 1) ? 0x1032u : 0x3210u;

        const int stop = min(units, seg.at + seg.e.units);
        for (; mine < stop; mine += WARPS) {
            const int st = done % STAGES;
            if (!dead && !mbar_wait_warp(&S.abort, &S.full[w][st], (unsigned)(done / STAGES) & 1u, P.status, 61)) dead = true;
            const Stage<ASYM>& X = S.ring[w][st];
            const unsigned valid = S.valid[w][st];
            const int tok0 = (seg.e.lo / UNIT + mine - seg.at) * UNIT;
            const bool plain = valid == 3u && tok0 >= all_lo && tok0 + UNIT <= all_hi;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                // sixteen tokens at a time
                float s[2][4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    s[b][0] = s[b][1] = s[b][2] = s[b][3] = 0.f;
                    const uint4 kw = *reinterpret_cast<const uint4*>(X.k + (16 * h + 8 * b + g) * KV_ROW + 16 * t);
                    const unsigned word[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        unsigned c[4];
                        codes_f16<ASYM>(word[i], c);
                        mma_f16(s[b], qa[2 * i], c[0], c[1]);
                        mma_f16(s[b], qa[2 * i + 1], c[2], c[3]);
                    }
                }
                // scores of this thread's row for tokens 2 t, 2 t + 1 of both groups of 8
                float z[4], vs[4], vl[4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int at = 16 * h + 8 * b + 2 * t;
                    float k0, k1, l0 = 0.f, l1 = 0.f;
                    if (ASYM) {
                        const float4 kk = *reinterpret_cast<const float4*>(X.ks + 8 * at), vv = *reinterpret_cast<const float4*>(X.vs + 8 * at);
                        k0 = kk.x; l0 = kk.y; k1 = kk.z; l1 = kk.w;
                        vs[2 * b] = vv.x; vl[2 * b] = vv.y; vs[2 * b + 1] = vv.z; vl[2 * b + 1] = vv.w;
                    } else {
                        const float2 kk = *reinterpret_cast<const float2*>(X.ks + 4 * at), vv = *reinterpret_cast<const float2*>(X.vs + 4 * at);
                        k0 = kk.x; k1 = kk.y;
                        vs[2 * b] = vv.x; vs[2 * b + 1] = vv.y;
                        vl[2 * b] = vl[2 * b + 1] = 0.f;
                    }
                    const float d0 = fmaf(s[b][2], 1.f / 2048.f, s[b][0]), d1 = fmaf(s[b][3], 1.f / 2048.f, s[b][1]);
                    z[2 * b] = d0 * (k0 * factor);
                    z[2 * b + 1] = d1 * (k1 * factor);
                    if (ASYM) {
                        z[2 * b] = fmaf(l0, qsum, z[2 * b]);
                        z[2 * b + 1] = fmaf(l1, qsum, z[2 * b + 1]);
                    }
                }
                if (!plain) {
                    const bool page = (valid >> h) & 1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int tok = tok0 + 16 * h + 8 * (i >> 1) + 2 * t + (i & 1);
                        if (!page || tok < row_lo || tok >= row_hi) {
                            z[i] = -INFINITY;
                            vs[i] = vl[i] = 0.f;
                        }
                    }
                }
                const float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
                if (__any_sync(0xffffffffu, top > m + MOVE)) {
                    float mx = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    mx = fmaxf(mx, m);
                    const float keep = mx == -INFINITY ? 1.f : ex2(m - mx);
                    m = mx;
                    l *= keep;
                    add *= keep;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        o[i][0] *= keep; o[i][1] *= keep; o[i][2] *= keep; o[i][3] *= keep;
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                unsigned pa[4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float p0 = ex2(z[2 * b] - base), p1 = ex2(z[2 * b + 1] - base);
                    l += p0 + p1;
                    if (ASYM) add = fmaf(p0, vl[2 * b], fmaf(p1, vl[2 * b + 1], add));
                    const float w0 = p0 * vs[2 * b], w1 = p1 * vs[2 * b + 1];
                    const __nv_bfloat162 hi = __floats2bfloat162_rn(w0, w1);
                    const float2 back = __bfloat1622float2(hi);
                    pa[2 * b] = __byte_perm(as_u(hi), 0, order);
                    pa[2 * b + 1] = __byte_perm(as_u(__floats2bfloat162_rn(w0 - back.x, w1 - back.y)), 0, order);
                }
                // values: coordinates 16 g .. of tokens 2 t, 2 t + 1 of both groups, the second one first where t is odd: a load then
                // takes two even and two odd rows, which lie in different halves of the banks
                const unsigned char* vp = X.v + (16 * h + 2 * t) * KV_ROW + 8 * g;
                const uint2 v0 = *reinterpret_cast<const uint2*>(vp + (t & 1) * KV_ROW), v1 = *reinterpret_cast<const uint2*>(vp + (~t & 1) * KV_ROW);
                const uint2 v2 = *reinterpret_cast<const uint2*>(vp + (8 + (t & 1)) * KV_ROW), v3 = *reinterpret_cast<const uint2*>(vp + (8 + (~t & 1)) * KV_ROW);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned sel = (i & 1) ? 0x7632u : 0x5410u;
                    unsigned c0[4], c1[4];
                    codes_bf16<ASYM>(__byte_perm(i < 2 ? v0.x : v0.y, i < 2 ? v1.x : v1.y, sel), c0);
                    codes_bf16<ASYM>(__byte_perm(i < 2 ? v2.x : v2.y, i < 2 ? v3.x : v3.y, sel), c1);
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma_bf16(o[4 * i + j], pa, c0[j], c1[j]);
                }
            }
            ++done;
            __syncwarp();
            if (!dead) issue();
        }

        // ---- the warps' sums ----
#pragma unroll
        for (int h = 1; h < 4; h <<= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, h);
            add += __shfl_xor_sync(0xffffffffu, add, h);
        }
        if (t == 0) {
            S.m[w][g] = m;
            S.l[w][g] = l;
            S.add[w][g] = add;
        }
        // thread (g, t): row g, coordinates 32 t .. 32 t + 31
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int i = 4 * (c & 3), k = c >> 2;
            const float4 x = make_float4(o[i][k] + o[i][k + 2], o[i + 1][k] + o[i + 1][k + 2], o[i + 2][k] + o[i + 2][k + 2], o[i + 3][k] + o[i + 3][k + 2]);
            *reinterpret_cast<float4*>(&S.part[w][g * 128 + 32 * t + 4 * (c ^ (lane & 7))]) = x;
        }
        __syncthreads();
        const bool starts = seg.at >= 0, ends = seg.at + seg.e.units <= units;
        if (w < 2) {
            const int row = 4 * w + (lane >> 3), l8 = lane & 7;
            float top = S.m[0][row];
#pragma unroll
            for (int i = 1; i < WARPS; ++i) top = fmaxf(top, S.m[i][row]);
            float y[16], total = 0.f, extra = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float keep = S.m[i][row] == -INFINITY && top == -INFINITY ? 1.f : ex2(S.m[i][row] - top);
                total = fmaf(S.l[i][row], keep, total);
                extra = fmaf(S.add[i][row], keep, extra);
#pragma unroll
                for (int q = 0; q < 4; ++q) {            // coordinates 64 (q >> 1) + 8 l8 + 4 (q & 1) ..
                    const int at = 64 * (q >> 1) + 8 * l8 + 4 * (q & 1), who = 4 * row + (at >> 5);
                    const float4 x = *reinterpret_cast<const float4*>(&S.part[i][row * 128 + (at & ~31) + 4 * (((at & 31) >> 2) ^ (who & 7))]);
                    y[4 * q] = fmaf(x.x, keep, y[4 * q]);
                    y[4 * q + 1] = fmaf(x.y, keep, y[4 * q + 1]);
                    y[4 * q + 2] = fmaf(x.z, keep, y[4 * q + 2]);
                    y[4 * q + 3] = fmaf(x.w, keep, y[4 * q + 3]);
                }
            }
            if (starts && ends) {
                const float by = total == 0.f ? 0.f : 1.f / total;
                kv_hadamard(y, l8);
                if (l8 == 0) y[0] = fmaf(extra, 128.f, y[0]);                // the transform of a row of `extra`
                if (seg.e.row0 + row < seg.e.rows) {
                    int token, head;
                    row_of(A, seg, row, token, head);
                    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + (seg.e.first + token) * A.out_token + head * A.out_head;
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] *= by * KV_NORM;
                    if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
                    if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
                }
            } else {
                float* part = P.parts + ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * PART;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(part + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                if (l8 == 0) {
                    part[ROWS * 128 + row] = top;
                    part[ROWS * 128 + ROWS + row] = total;
                    part[ROWS * 128 + 2 * ROWS + row] = extra;
                }
                if (threadIdx.x == 0 && starts) {
                    const int beyond = seg.at + seg.e.units - units;
                    P.joins[blockIdx.x] = KvJoin{seg.index, seg.head, 1 + (beyond + units - 1) / units, 0};   // the blocks behind have as many units, or their rest
                }
            }
        }
        if (seg.at + seg.e.units >= units) break;
        kv_next(A, seg, P.line.entries, P.line.tiles, ROWS, UNIT);
    }
    if (dead) drain_copies(S.full[w], STAGES, fetched);
}

// The segments that several blocks share: block b joins the one that starts in block b, eight lanes a row.
__global__ __launch_bounds__(64) void k_kv_attn_join(const __grid_constant__ Args P)
{
    kv_wait_before();
    kv_let_next();
    const KvJoin j = P.joins[blockIdx.x];
    if (j.blocks == 0) return;
    const gbs_kv_attn& A = P.a;
    KvSeg s;
    s.index = j.index;
    s.head = j.head;
    s.e = kv_entry(A, j.index, P.line.tiles, ROWS, UNIT);
    const int row = threadIdx.x >> 3, l8 = threadIdx.x & 7;
    float top = -INFINITY, total = 0.f, extra = 0.f, y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0.f;
    for (int b = 0; b < j.blocks; ++b) {
        const float* part = P.parts + ((long long)(blockIdx.x + b) * 2 + (b == 0 ? 1 : 0)) * PART;
        const float m = part[ROWS * 128 + row], mx = fmaxf(m, top);
        const float keep = mx == -INFINITY ? 1.f : ex2(top - mx), more = mx == -INFINITY ? 1.f : ex2(m - mx);
        top = mx;
        total = total * keep + part[ROWS * 128 + ROWS + row] * more;
        extra = extra * keep + part[ROWS * 128 + 2 * ROWS + row] * more;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 x = *reinterpret_cast<const float4*>(part + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1));
            y[4 * q] = fmaf(x.x, more, y[4 * q] * keep);
            y[4 * q + 1] = fmaf(x.y, more, y[4 * q + 1] * keep);
            y[4 * q + 2] = fmaf(x.z, more, y[4 * q + 2] * keep);
            y[4 * q + 3] = fmaf(x.w, more, y[4 * q + 3] * keep);
        }
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
    kv_hadamard(y, l8);
    if (l8 == 0) y[0] = fmaf(extra, 128.f, y[0]);
    if (s.e.row0 + row >= s.e.rows) return;
    int token, head;
    row_of(A, s, row, token, head);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + (s.e.first + token) * A.out_token + head * A.out_head;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] *= by * KV_NORM;
    if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
    if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
}

int blocks_of(const gbs_plan* p) { return p->sm_count * BLOCKS_PER_SM; }

}  // namespace

int64_t gbs_kv_attn_workspace(const gbs_plan* p, int, int)
{
    return (int64_t)blocks_of(p) * (2 * PART * sizeof(float) + sizeof(KvJoin)) + 16;
}

int gbs_kv_attn_launch(const gbs_plan* p, const gbs_kv_attn& A, void* workspace, cudaStream_t stream)
{
    Args P = {};
    P.a = A;
    P.line.tile_rows = ROWS;
    P.line.unit = UNIT;
    P.line.tiles = (int)(((int64_t)A.max_tokens * A.group + ROWS - 1) / ROWS);
    P.line.entries = A.n_items * P.line.tiles;
    P.line.least = 2 * WARPS;
    const int blocks = blocks_of(p);
    P.joins = static_cast<KvJoin*>(workspace);
    P.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + blocks * sizeof(KvJoin));
    P.status = p->d_status;
    const size_t smem = p->asym ? sizeof(Smem<true>) : sizeof(Smem<false>);
    const void* f = p->asym ? (const void*)k_kv_attn_few<true> : (const void*)k_kv_attn_few<false>;
    const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    const int rc = gbs_kv_launch(p, p->asym ? k_kv_attn_few<true> : k_kv_attn_few<false>, dim3((unsigned)blocks), THREADS, smem, stream, P);
    if (rc != 0) return rc;
    return gbs_kv_launch(p, k_kv_attn_join, dim3((unsigned)blocks), 64, 0, stream, P);
}
