// Attention over the paged KV cache for few query rows (gbs_kv_attention: decoding).
//
// With khat = Delta c (+ lo) in the rotated basis, scores are Delta_k (H q . c) (+ lo sum H q) and the result is H sum_j (p_j Delta_v) c_j, or
// H (sum_j (p_j Delta_v) (c_j - 8) + sum_j p_j mid_j) with mid = lo + 8 Delta: the codes go into the matrix unit as they are, exactly, and the rotation is applied to eight query rows and
// eight results instead of to every cached row.
//
// What bounds it is the cache, 136 or 144 bytes a token and KV head, read once, and next to it the conversion of 256 codes a token.
// The codes are the tall operand of both products (16 tokens, then 16 coordinates, by 8 query rows), so no row of the matrix unit is idle.
// Scores are integers: key codes are bytes after a mask and a shift (3 operations for 8 codes), and a query row is an integer of 16 bits
// per coordinate, in two pieces of 8; sums are exact, and the offset 8 of symmetric codes is the value that they start from.  Weights span too many binary places for that:
// values become fp16 (a nibble in the mantissa of 1024, which is subtracted again, exactly; 9 operations for 8 codes).  In fp16 for both products, with
// the weights in two pieces as well, a unit took 797 instructions instead of 576, and 16 sequences x 32 KV heads x 4096 tokens of one query row 107 us instead of 72: 4.2 TB/s of
// the cache, two thirds of a plain copy's rate.  What bounds it then is latency: issue slots are 54 % used, the integer pipe 47 %, DRAM 52 %; 128 registers and
// 160 threads leave 15 warps an SM, each a chain of loads, integer products, scores, weights and products again.
// Layouts are chosen so that codes go from shared memory to the operand registers without being moved between threads: the order of the 128
// coordinates of a score, of a group's 16 tokens and of the 128 rows of the result is free, as long as both operands have the same.
// Only the weights are transposed on the way (movmatrix).
//
// Two running maxima: m of the scores z (log2), as in any softmax, and M of z + log2 Delta_v, which keeps w inside fp16 whatever the
// sizes of the values: w = 2^(z - m) Delta_v 2^(m - M).  They are moved only when a score exceeds m by 8 or w its range, which is rare.
//
// One warp of a block fetches units of 32 tokens (bulk copies into a ring), four at a time, eight lanes for the up to eight pieces of one.  The
// others take them in turn, keep sums for their tokens in registers, and meet where a segment ends.
#include <stddef.h>

#include <algorithm>

#include "gbs_kv_attn.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int ROWS = 8, UNIT = 32;
constexpr int WARPS = 4, THREADS = 32 * WARPS + 32;  // warps that compute, and the one that fetches
constexpr int STAGES = 12;                           // unit i of a block's is worked on by warp i % WARPS, from stage i % STAGES
// A stage is always the same warp's.  A wait for a phase goes by its parity, so it is one only for who has seen the phase before end; another warp, ahead
// of the one whose copy is late, would read the stage at once.
static_assert(STAGES % WARPS == 0, "a stage has one warp");
constexpr int PART = KV_PART<ROWS>;
static_assert(2 * WARPS == ROWS, "each warp finishes two rows");
constexpr int BLOCKS_PER_SM = 3;
constexpr float MOVE = 8.f;                          // m moves when a score is so much (log2) above it
constexpr float W_MOST = 32768.f;                    // M moves when a w is beyond that

template <bool ASYM>
struct Stage {
    static constexpr int SCALE = UNIT * (ASYM ? 8 : 4);
    unsigned char k[UNIT * KV_ROW], v[UNIT * KV_ROW];
    unsigned char ks[SCALE], vs[SCALE];
};

template <bool ASYM>
struct Smem {
    Stage<ASYM> ring[STAGES];
    float part[WARPS][ROWS * 128];                   // 16-byte pieces c of each 64 bytes of rows 2 t, 2 t + 1 at c ^ t
    // of two segments in turn: the rows' integers (upper and lower byte; of 8 coordinates the even ones first), their factors and sums, what
    // each row sees and what all of them see, the segment and the block's piece of it
    struct alignas(16) Query {
        signed char h[ROWS][128], l[ROWS][128];
        float factor[ROWS];
        int sum[ROWS], lo[ROWS], hi[ROWS];
        int all_lo, all_hi;
        KvSeg seg;
        KvPiece piece;
        bool last;
        // where the integers were, at the segment's end: the warps' maxima m, totals, sums of p mid, and maxima M
        __device__ __forceinline__ float* stat(int which, int warp) { return reinterpret_cast<float*>(h) + (which * WARPS + warp) * ROWS; }
    } query[2];
    static_assert(4 * WARPS * ROWS * sizeof(float) <= sizeof(Query::h), "room for the warps' statistics");
    unsigned long long full[STAGES], empty[STAGES], qfull[2], qempty[2];
    unsigned valid[STAGES];                          // bit h: tokens 16 h .. of the unit have a page
    KvSeg seg;                                       // the block's first segment
    long long share[WARPS + 1];
    int abort;
};

static_assert(offsetof(Smem<true>, query) % 16 == 0 && offsetof(Smem<false>, query) % 16 == 0 && sizeof(Smem<true>::Query) % 16 == 0, "read 16 bytes at a time");
static_assert(sizeof(Smem<true>) + 1024 <= 228 * 1024 / BLOCKS_PER_SM, "so many blocks have room on an SM");
static_assert(sizeof(Stage<true>) % 128 == 0 && sizeof(Stage<false>) % 128 == 0, "copied and read 16 bytes at a time");

__device__ __forceinline__ void mma_f16(float c[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, const unsigned b[2])
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_u8(int c[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, const unsigned b[2])
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
// 8 x 8 16-bit numbers, a row in four lanes: rows become columns
__device__ __forceinline__ unsigned transposed(unsigned x)
{
    unsigned y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The query rows of a segment by one warp, eight lanes a row: rotated, and made integers.
template <bool ASYM>
__device__ __forceinline__ void prepare(const gbs_kv_attn& A, const KvSeg& seg, typename Smem<ASYM>::Query& Q, int lane)
{
    const int l8 = lane & 7;
    uint4 raw[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = 4 * r + (lane >> 3);
        raw[r][0] = raw[r][1] = make_uint4(0, 0, 0, 0);
        if (seg.e.row0 + row < seg.e.rows) {
            int token, head;
            kv_row_of(A, seg, row, token, head);
            const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(A.q) + (seg.e.first + token) * A.q_token + head * A.q_head;
            if (8 * l8 < A.d) raw[r][0] = *reinterpret_cast<const uint4*>(x + 8 * l8);
            if (64 + 8 * l8 < A.d) raw[r][1] = *reinterpret_cast<const uint4*>(x + 64 + 8 * l8);
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = 4 * r + (lane >> 3);
        float y[16];
        kv_unpack_bf16(raw[r][0], y);
        kv_unpack_bf16(raw[r][1], y + 8);
        kv_hadamard(y, l8);
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(y[i]));
#pragma unroll
        for (int h = 1; h < 8; h <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, h));
        // integers of up to 32512, whose upper byte is at most 127; a row that is not finite has a factor that is not a number
        const float up = m < 1e-30f ? 1.2379400392853803e27f : 1.f;     // 2^90
        const float by = m > 0.f ? 32512.f / (m * up) : 0.f;
        int q[16], sum = 0;
        float wrong = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            q[i] = __float2int_rn(fminf(fmaxf(y[i] * up * by, -32512.f), 32512.f));
            sum += q[i];
            wrong += y[i] * 0.f;
        }
#pragma unroll
        for (int h = 1; h < 8; h <<= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, h);
            wrong += __shfl_xor_sync(0xffffffffu, wrong, h);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            unsigned high[2] = {0, 0}, low[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int x = q[8 * half + i], top = (x + 128) >> 8;
                high[i & 1] |= (unsigned)(top & 255) << (8 * (i >> 1));
                low[i & 1] |= (unsigned)((x - 256 * top) & 255) << (8 * (i >> 1));
            }
            *reinterpret_cast<uint2*>(&Q.h[row][64 * half + 8 * l8]) = make_uint2(high[0], high[1]);
            *reinterpret_cast<uint2*>(&Q.l[row][64 * half + 8 * l8]) = make_uint2(low[0], low[1]);
        }
        if (l8 == 0) {
            Q.factor[row] = m * (A.scale * (KV_NORM * 1.4426950408889634f / 32512.f)) + wrong;
            Q.sum[row] = sum;
            const int token = A.by_group(min(seg.e.row0 + row, seg.e.rows - 1));
            Q.lo[row] = kv_row_lo(A, seg.e, token);
            Q.hi[row] = kv_row_hi(A, seg.e, token);
            if (row == 0) {                          // the last row sees the latest window, the first the shortest past
                Q.all_lo = kv_row_lo(A, seg.e, A.by_group(min(seg.e.rows, seg.e.row0 + ROWS) - 1));
                Q.all_hi = Q.hi[0];
            }
        }
    }
}

// An infinite scale becomes NaN: a score of -infinity is a masked one.
__device__ __forceinline__ float no_inf(float x) { return fmaf(x, 0.f, x); }

// the warps that compute
__device__ __forceinline__ void meet() { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); }
// The same, and whether any of their threads says so (a barrier of its own: one that is waited for in both ways has to be at rest between them).
__device__ __forceinline__ bool meet_any(bool x)
{
    int any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.or.pred q, 2, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((int)x), "n"(32 * WARPS) : "memory");
    return any != 0;
}

template <bool ASYM, bool TEST>
__global__ __launch_bounds__(THREADS, BLOCKS_PER_SM) void k_kv_attn_few(const __grid_constant__ KvAttnArgs P)
{
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Smem<ASYM>& S = *reinterpret_cast<Smem<ASYM>*>(smem_raw);
    const gbs_kv_attn& A = P.a;
    const int lane = threadIdx.x & 31, w = warp_index(), g = lane >> 2, t = lane & 3;
    if (threadIdx.x == 0) S.abort = 0;
    if (threadIdx.x < STAGES) {
        mbar_init(&S.full[threadIdx.x], 1);
        mbar_init(&S.empty[threadIdx.x], 1);
    }
    if (threadIdx.x < 2) {
        mbar_init(&S.qfull[threadIdx.x], 1);
        mbar_init(&S.qempty[threadIdx.x], WARPS);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    kv_wait_before();
    kv_let_next();

    const int places = kv_share<THREADS>(A, P.line, &S.seg, S.share);
    if (threadIdx.x == 0 && P.line.pad >= 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};
    if (places == 0) return;

    if (w == WARPS) {
        // ---- fetching ----
        const int ps_log = A.c.page_log, T = min(UNIT, 1 << ps_log);
        const int mine = lane >> 3, half = (lane >> 2) & 1, piece = lane & 3;
        const bool copies = T < UNIT || half == 0;           // this lane copies a piece
        const unsigned piece_bytes = piece < 2 ? T * KV_ROW : T * (ASYM ? 8 : 4);
        const int in_block = piece < 2 ? piece * (KV_ROW << ps_log) : (2 * KV_ROW << ps_log) + (piece - 2) * ((ASYM ? 8 : 4) << ps_log);
        const int in_slot = piece < 2 ? KV_ROW : (ASYM ? 8 : 4);
        const int in_stage = (piece < 2 ? piece * UNIT * KV_ROW : 2 * UNIT * KV_ROW + (piece - 2) * Stage<ASYM>::SCALE) + half * (int)piece_bytes;
        bool dead = false, more = true;
        int at = 0, armed = 0;                               // units of the segments so far, and of all that have been sent for
        KvSeg seg = S.seg;
        for (int round = 0; more && !dead; ++round) {
            const KvPiece part = kv_piece(P.line, seg, places);
            more = kv_more(P.line, seg, places);
            const int* row = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            const int off = seg.head * A.c.block_bytes + in_block;
            int tok = ((seg.e.lo >> 5) + part.skip + mine) * UNIT + half * 16;
            int page = copies && mine < part.n && tok < seg.e.hi ? row[tok >> ps_log] : -1;
            for (int i = 0; i < part.n || i == 0; i += 4) {
                const int u = at + i + mine, st = u % STAGES, use = u / STAGES;
                const bool have = i + mine < part.n;
                const int next_tok = tok + 4 * UNIT, next = copies && i + 4 + mine < part.n && next_tok < seg.e.hi ? row[next_tok >> ps_log] : -1;
                if (have && use > 0 && (kv_lost<TEST>(P, &S.abort, 62, round) || !mbar_wait(&S.abort, &S.empty[st], (unsigned)(use - 1) & 1u, P.status, 62))) dead = true;
                if (__any_sync(0xffffffffu, dead)) { dead = true; break; }
                const bool ok = have && (unsigned)page < (unsigned)A.c.n_pages;
                const unsigned who = __ballot_sync(0xffffffffu, ok) >> (8 * mine), first = who & 1, second = (who >> 4) & 1;
                if (have && (lane & 7) == 0) {
                    S.valid[st] = T == UNIT ? 3u * first : first | second << 1;
                    mbar_arrive_expect_tx(&S.full[st], (first + second) * (unsigned)(T * (2 * KV_ROW + (ASYM ? 16 : 8))));
                }
                __syncwarp();
                if (ok)
                    bulk_load(reinterpret_cast<unsigned char*>(&S.ring[st]) + in_stage,
                              A.c.pages + ((long long)page * A.c.page_bytes + off + (tok & ((1 << ps_log) - 1)) * in_slot), piece_bytes, &S.full[st]);
                armed = at + max(min(i + 4, part.n), 0);
                tok = next_tok;
                page = next;
                if (i > 0) continue;
                // with the first units under way: the segment's query rows, eight lanes a row, rotated and made integers
                if (round > 1 && (kv_lost<TEST>(P, &S.abort, 63, round) || !mbar_wait_warp(&S.abort, &S.qempty[round & 1], (unsigned)(round / 2 - 1) & 1u, P.status, 63))) {
                    dead = true;
                    break;
                }
                prepare<ASYM>(A, seg, S.query[round & 1], lane);
                if (lane == 0) {
                    S.query[round & 1].seg = seg;
                    S.query[round & 1].piece = part;
                    S.query[round & 1].last = !more;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.qfull[round & 1]);
            }
            at += max(part.n, 0);
            if (more) kv_next(A, P.line, seg);
        }
        // The others may have given up on copies that are still on their way: in the self-test, where they leave at once.  A wait that ran out by itself
        // began two seconds ago; what had been sent for by then is not on its way any more.  (Always: 64 ragged sequences 37.9 us -> 38.4.)
        if (dead || TEST) drain_copies(S.full, STAGES, armed);
        return;
    }

    // ---- the segments ----
    int mine = w, st = w, done = 0;                          // this warp's next unit of the block's, and its stage; units of the segments before
    unsigned phase = 0;
    for (int round = 0;; ++round) {
        auto& Q = S.query[round & 1];
        // a warp whose wait ran out goes on to where the warps meet, and there all of them leave: what Q holds then counts for nothing
        bool dead = kv_lost<TEST>(P, &S.abort, 64, round) || !mbar_wait_warp(&S.abort, &S.qfull[round & 1], (unsigned)(round / 2) & 1u, P.status, 64);
        unsigned qh[4][2], ql[4][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 h = *reinterpret_cast<const uint4*>(&Q.h[g][32 * t + 16 * i]), l = *reinterpret_cast<const uint4*>(&Q.l[g][32 * t + 16 * i]);
            qh[2 * i][0] = h.x; qh[2 * i][1] = h.y; qh[2 * i + 1][0] = h.z; qh[2 * i + 1][1] = h.w;
            ql[2 * i][0] = l.x; ql[2 * i][1] = l.y; ql[2 * i + 1][0] = l.z; ql[2 * i + 1][1] = l.w;
        }
        // this thread's scores and results are of rows 2 t and 2 t + 1
        const float2 factor = *reinterpret_cast<const float2*>(&Q.factor[2 * t]);
        const int2 qsum = *reinterpret_cast<const int2*>(&Q.sum[2 * t]);
        const int from0 = ASYM ? 0 : -8 * qsum.x, from1 = ASYM ? 0 : -8 * qsum.y;
        const float lift0 = (float)qsum.x * factor.x, lift1 = (float)qsum.y * factor.y;
        float o[8][4];                                   // (coordinate 16 g + 2 j, rows 2 t, 2 t + 1), (coordinate 16 g + 2 j + 1, the same)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        float m0 = NONE, m1 = NONE, mw0 = NONE, mw1 = NONE, up0 = 0.f, up1 = 0.f, l0 = 0.f, l1 = 0.f, add0 = 0.f, add1 = 0.f;     // up = 64 2^(m - M)

        const int stop = dead ? done : done + max(Q.piece.n, 0), tok_at = ((Q.seg.e.lo >> 5) + Q.piece.skip - done) * UNIT;
        for (; mine < stop; mine += WARPS) {
            if (kv_lost<TEST>(P, &S.abort, 61, round) || !mbar_wait_warp(&S.abort, &S.full[st], phase, P.status, 61)) {
                dead = true;
                break;
            }
            const Stage<ASYM>& X = S.ring[st];
            const unsigned valid = S.valid[st];
            const int tok0 = tok_at + mine * UNIT;
            const bool plain = valid == 3u && tok0 >= Q.all_lo && tok0 + UNIT <= Q.all_hi;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                // sixteen tokens at a time
                // row g of an operand is token g ^ ((g >> 1) & 1), row g + 8 the one 8 further: see the values
                const int tg = 16 * h + (g ^ ((g >> 1) & 1));
                const uint4 ka = *reinterpret_cast<const uint4*>(X.k + tg * KV_ROW + 16 * t), kb = *reinterpret_cast<const uint4*>(X.k + (tg + 8) * KV_ROW + 16 * t);
                const unsigned wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
                int s[4] = {0, 0, 0, 0}, r[4] = {from0, from1, from0, from1};
                constexpr unsigned FLIP = ASYM ? 0u : 0x08080808u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned a0 = kv_and_xor(wa[i], 0x0f0f0f0fu, FLIP), a1 = kv_and_xor(wb[i], 0x0f0f0f0fu, FLIP);
                    const unsigned a2 = kv_and_xor(wa[i] >> 4, 0x0f0f0f0fu, FLIP), a3 = kv_and_xor(wb[i] >> 4, 0x0f0f0f0fu, FLIP);
                    mma_u8(s, a0, a1, a2, a3, qh[i]);
                    mma_u8(r, a0, a1, a2, a3, ql[i]);
                }
                float f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = (float)(256 * s[i] + r[i]);
                float va, vb, la = 0.f, lb = 0.f, z[4];  // Delta and mid; (token, row 2 t), (token, row 2 t + 1), (token + 8, the same)
                if (ASYM) {
                    const float2 sa = *reinterpret_cast<const float2*>(X.ks + 8 * tg), sb = *reinterpret_cast<const float2*>(X.ks + 8 * (tg + 8));
                    const float2 ua = *reinterpret_cast<const float2*>(X.vs + 8 * tg), ub = *reinterpret_cast<const float2*>(X.vs + 8 * (tg + 8));
                    const float ka = no_inf(fmaf(sa.y, 0.f, sa.x)), kb = no_inf(fmaf(sb.y, 0.f, sb.x));
                    z[0] = fmaf(f[0], ka * factor.x, sa.y * lift0);
                    z[1] = fmaf(f[1], ka * factor.y, sa.y * lift1);
                    z[2] = fmaf(f[2], kb * factor.x, sb.y * lift0);
                    z[3] = fmaf(f[3], kb * factor.y, sb.y * lift1);
                    va = fmaf(ua.y, 0.f, ua.x); la = fmaf(8.f, ua.x, ua.y); vb = fmaf(ub.y, 0.f, ub.x); lb = fmaf(8.f, ub.x, ub.y);
                } else {
                    const float sa = no_inf(*reinterpret_cast<const float*>(X.ks + 4 * tg)), sb = no_inf(*reinterpret_cast<const float*>(X.ks + 4 * (tg + 8)));
                    va = *reinterpret_cast<const float*>(X.vs + 4 * tg);
                    vb = *reinterpret_cast<const float*>(X.vs + 4 * (tg + 8));
                    z[0] = f[0] * (sa * factor.x);
                    z[1] = f[1] * (sa * factor.y);
                    z[2] = f[2] * (sb * factor.x);
                    z[3] = f[3] * (sb * factor.y);
                }
                if (!plain) {
                    const bool page = (valid >> h) & 1;
                    const int2 lo = *reinterpret_cast<const int2*>(&Q.lo[2 * t]), hi = *reinterpret_cast<const int2*>(&Q.hi[2 * t]);
                    const int ta = tok0 + tg, tb = ta + 8;
                    if (!page || ta < lo.x || ta >= hi.x) z[0] = -INFINITY;
                    if (!page || ta < lo.y || ta >= hi.y) z[1] = -INFINITY;
                    if (!page || tb < lo.x || tb >= hi.x) z[2] = -INFINITY;
                    if (!page || tb < lo.y || tb >= hi.y) z[3] = -INFINITY;
                    // scales that are no numbers make the scores of the rows that see them none, and those of tokens that no row sees may be anything
                    if ((z[0] == -INFINITY && z[1] == -INFINITY) || !(fabsf(va) < INFINITY) || !(fabsf(la) < INFINITY)) {
                        if (z[0] != -INFINITY) z[0] = NAN;
                        if (z[1] != -INFINITY) z[1] = NAN;
                        va = la = 0.f;
                    }
                    if ((z[2] == -INFINITY && z[3] == -INFINITY) || !(fabsf(vb) < INFINITY) || !(fabsf(lb) < INFINITY)) {
                        if (z[2] != -INFINITY) z[2] = NAN;
                        if (z[3] != -INFINITY) z[3] = NAN;
                        vb = lb = 0.f;
                    }
                }
                float p[4], x[4];
                auto weigh = [&]() {
                    p[0] = kv_ex2(z[0] - m0);
                    p[1] = kv_ex2(z[1] - m1);
                    p[2] = kv_ex2(z[2] - m0);
                    p[3] = kv_ex2(z[3] - m1);
                    x[0] = p[0] * (va * up0);
                    x[1] = p[1] * (va * up1);
                    x[2] = p[2] * (vb * up0);
                    x[3] = p[3] * (vb * up1);
                };
                weigh();
                if (__any_sync(0xffffffffu, fmaxf(z[0], z[2]) > m0 + MOVE || fmaxf(z[1], z[3]) > m1 + MOVE || fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) > W_MOST)) {
                    const float ga = __log2f(va), gb = __log2f(vb);
                    float t0 = fmaxf(z[0], z[2]), t1 = fmaxf(z[1], z[3]), u0 = fmaxf(z[0] + ga, z[2] + gb), u1 = fmaxf(z[1] + ga, z[3] + gb);
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) {
                        t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, k));
                        t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, k));
                        u0 = fmaxf(u0, __shfl_xor_sync(0xffffffffu, u0, k));
                        u1 = fmaxf(u1, __shfl_xor_sync(0xffffffffu, u1, k));
                    }
                    t0 = fmaxf(t0, m0);
                    t1 = fmaxf(t1, m1);
                    u0 = fmaxf(u0, mw0);
                    u1 = fmaxf(u1, mw1);
                    const float k0 = kv_ex2(m0 - t0), k1 = kv_ex2(m1 - t1), y0 = kv_ex2(mw0 - u0), y1 = kv_ex2(mw1 - u1);
                    m0 = t0; m1 = t1; mw0 = u0; mw1 = u1;
                    up0 = W_UP * kv_ex2(fminf(m0 - mw0, 100.f));                // no values but zeros: M stays where it was
                    up1 = W_UP * kv_ex2(fminf(m1 - mw1, 100.f));
                    l0 *= k0; l1 *= k1; add0 *= k0; add1 *= k1;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        o[i][0] *= y0; o[i][1] *= y1; o[i][2] *= y0; o[i][3] *= y1;
                    }
                    weigh();
                }
                l0 += p[0] + p[2];
                l1 += p[1] + p[3];
                if (ASYM) {
                    add0 = fmaf(p[0], la, fmaf(p[2], lb, add0));
                    add1 = fmaf(p[1], la, fmaf(p[3], lb, add1));
                }
                const unsigned b[2] = {transposed(as_u(__floats2half2_rn(x[0], x[1]))), transposed(as_u(__floats2half2_rn(x[2], x[3])))};
                // values: coordinates 16 g .. of the tokens that rows 2 t, 2 t + 1 (and 8 further) stand for, in their order: a load
                // takes two even and two odd tokens, which lie in different halves of the banks
                const unsigned char* vp = X.v + (16 * h + 2 * t) * KV_ROW + 8 * g;
                const uint2 v0 = *reinterpret_cast<const uint2*>(vp + (t & 1) * KV_ROW), v1 = *reinterpret_cast<const uint2*>(vp + (~t & 1) * KV_ROW);
                const uint2 v2 = *reinterpret_cast<const uint2*>(vp + (8 + (t & 1)) * KV_ROW), v3 = *reinterpret_cast<const uint2*>(vp + (8 + (~t & 1)) * KV_ROW);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned sel = (i & 1) ? 0x7632u : 0x5410u;
                    unsigned c[4], e[4];
                    kv_codes_f16<ASYM>(__byte_perm(i < 2 ? v0.x : v0.y, i < 2 ? v1.x : v1.y, sel), c);
                    kv_codes_f16<ASYM>(__byte_perm(i < 2 ? v2.x : v2.y, i < 2 ? v3.x : v3.y, sel), e);
                    mma_f16(o[2 * i], c[0], c[1], e[0], e[1], b);
                    mma_f16(o[2 * i + 1], c[2], c[3], e[2], e[3], b);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.empty[st]);
            if ((st += WARPS) >= STAGES) {
                st -= STAGES;
                phase ^= 1u;
            }
        }

        done = stop;
        // ---- the warps' sums ----
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, k);
            l1 += __shfl_xor_sync(0xffffffffu, l1, k);
            add0 += __shfl_xor_sync(0xffffffffu, add0, k);
            add1 += __shfl_xor_sync(0xffffffffu, add1, k);
        }
        const KvSeg seg = Q.seg;
        const KvPiece piece = Q.piece;
        const bool last = Q.last;
        meet();                                              // the sums before these have been read, and the integers of this segment's rows
        if (g == 0) {
            *reinterpret_cast<float2*>(Q.stat(0, w) + 2 * t) = make_float2(m0, m1);
            *reinterpret_cast<float2*>(Q.stat(1, w) + 2 * t) = make_float2(l0, l1);
            *reinterpret_cast<float2*>(Q.stat(2, w) + 2 * t) = make_float2(add0, add1);
            *reinterpret_cast<float2*>(Q.stat(3, w) + 2 * t) = make_float2(mw0, mw1);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float* to = &S.part[w][2 * t * 128 + 16 * g + 4 * (c ^ t)];
            *reinterpret_cast<float4*>(to) = make_float4(o[2 * c][0], o[2 * c][2], o[2 * c + 1][0], o[2 * c + 1][2]);
            *reinterpret_cast<float4*>(to + 128) = make_float4(o[2 * c][1], o[2 * c][3], o[2 * c + 1][1], o[2 * c + 1][3]);
        }
        if (meet_any(dead)) break;
        // two rows a warp, eight lanes a row (the upper half of the warp does the same and writes nothing)
        if (piece.n > 0) {
            const int row = 2 * w + ((lane >> 3) & 1), l8 = lane & 7;
            float top = NONE, top_w = NONE;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                top = fmaxf(top, Q.stat(0, i)[row]);
                top_w = fmaxf(top_w, Q.stat(3, i)[row]);
            }
            float y[16], total = 0.f, extra = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float keep = kv_ex2(Q.stat(0, i)[row] - top), keep_w = kv_ex2(Q.stat(3, i)[row] - top_w);
                total = fmaf(Q.stat(1, i)[row], keep, total);
                extra = fmaf(Q.stat(2, i)[row], keep, extra);
#pragma unroll
                for (int q = 0; q < 4; ++q) {            // coordinates 64 (q >> 1) + 8 l8 + 4 (q & 1) ..
                    const int at = 64 * (q >> 1) + 8 * l8 + 4 * (q & 1);
                    const float4 x = *reinterpret_cast<const float4*>(&S.part[i][row * 128 + (at & ~15) + 4 * (((at >> 2) & 3) ^ (row >> 1))]);
                    y[4 * q] = fmaf(x.x, keep_w, y[4 * q]);
                    y[4 * q + 1] = fmaf(x.y, keep_w, y[4 * q + 1]);
                    y[4 * q + 2] = fmaf(x.z, keep_w, y[4 * q + 2]);
                    y[4 * q + 3] = fmaf(x.w, keep_w, y[4 * q + 3]);
                }
            }
            if (piece.starts && piece.ends) {
                kv_finish(y, l8, top, top_w, total, extra);
                if (seg.e.row0 + row < seg.e.rows && lane < 16) {
                    int token, head;
                    kv_row_of(A, seg, row, token, head);
                    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + (seg.e.first + token) * A.out_token + head * A.out_head;
                    if (8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 8 * l8) = kv_pack_bf16(y);
                    if (64 + 8 * l8 < A.d) *reinterpret_cast<uint4*>(out + 64 + 8 * l8) = kv_pack_bf16(y + 8);
                }
            } else if (lane < 16) {
                float* part = P.parts + ((long long)blockIdx.x * 2 + (piece.starts ? 1 : 0)) * PART;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(part + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                if (l8 == 0) {
                    part[ROWS * 128 + row] = top;
                    part[ROWS * 128 + ROWS + row] = total;
                    part[ROWS * 128 + 2 * ROWS + row] = extra;
                    part[ROWS * 128 + 3 * ROWS + row] = top_w;
                }
                if (threadIdx.x == 0 && piece.starts) P.joins[blockIdx.x] = kv_join(P.line, seg, places);
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.qempty[round & 1]);
        if (last) break;
    }
}

int blocks_of(const gbs_plan* p) { return p->sm_count * BLOCKS_PER_SM; }

}  // namespace

int64_t gbs_kv_few_workspace(const gbs_plan* p)
{
    return (int64_t)blocks_of(p) * (2 * PART * sizeof(float) + sizeof(KvJoin)) + 16;
}

int gbs_kv_few_launch(const gbs_plan* p, const gbs_kv_attn& A, void* workspace, cudaStream_t stream)
{
    KvAttnArgs P = {};
    P.a = A;
    P.line.tile_rows = ROWS;
    P.line.unit_log = 5;
    P.line.tiles = (int)(((int64_t)A.max_tokens * A.group + ROWS - 1) / ROWS);
    P.line.by_tiles.set((unsigned)P.line.tiles);
    P.line.entries = A.n_items * P.line.tiles;
    // a short sequence is not worth dividing: the join's launch takes as long as a block needs for 16 units
    P.line.pad = A.max_len <= 16 * UNIT ? -1 : 7;
    P.line.least = P.line.pad < 0 ? 1 : 12;
    const int blocks = P.line.pad < 0 ? (int)std::min<int64_t>((int64_t)P.line.entries * A.c.heads, blocks_of(p)) : blocks_of(p);
    P.joins = static_cast<KvJoin*>(workspace);
    P.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + blocks * sizeof(KvJoin));
    P.status = p->d_status;
    const size_t smem = p->asym ? sizeof(Smem<true>) : sizeof(Smem<false>);
    const auto f = A.lost_code ? (p->asym ? k_kv_attn_few<true, true> : k_kv_attn_few<false, true>)
                               : (p->asym ? k_kv_attn_few<true, false> : k_kv_attn_few<false, false>);
    const cudaError_t e = cudaFuncSetAttribute((const void*)f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    const int rc = gbs_kv_launch(p, f, dim3((unsigned)blocks), THREADS, smem, stream, P);
    if (rc != 0 || P.line.pad < 0) return rc;
    return gbs_kv_launch(p, k_kv_attn_join<ROWS>, dim3((unsigned)blocks), 256, 0, stream, P);
}
