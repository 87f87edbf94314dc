// The weights that cached tokens get from many query rows (gbs_kv_attention_mass), on tcgen05: as in gbs_kv_mass.cu, one pass over the keys for the rows'
// sums, a second one for the tokens'.
//
// A query row is an integer of 22 bits per coordinate and sign, in two pieces of 11 that fp16 holds exactly, and so are the codes: every sum of 128 products is an integer below
// 2^22, exact in fp32 whatever the order, and 2048 times the upper one plus the lower one is the score's integer, rounded once.
//
// First pass (k_tc_kvmass_rows): rows are lanes, tokens columns.  A block has 128 rows against units of 128 tokens; a thread has a row and a part of a unit's
// tokens, with a maximum and a sum of its own.  Second pass (k_tc_kvmass_tokens): tokens are lanes, rows columns, so that what a token
// gets stays in one thread.  A block has pairs of units, whose codes are converted once, and goes over all tiles of 64 rows that see them.
// In both, sixteen warps take the scores from tensor memory, four turn codes into fp16, one issues the MMAs, one fetches query rows.  (Eight readers: 77 and 124 us instead of 71 and
// 102 for 1000 tokens of 4 query heads a KV head behind 5000, d = 80.)
// That now takes 64 and 69 us; the MMAs would take 20 and 22, ex2 as much.  Without any work on the scores 42 and 66 were left: a product of 128 x 128 takes its operands from shared
// memory at 128 bytes a cycle, all that there is, beside which codes and query rows are written there and factors read.  Issue slots are 46 and 49 % used, the tensor pipe 35 %.
#include <algorithm>

#include "gbs_kv_attn.cuh"
#include "gbs_tc_common.cuh"

namespace {

constexpr int UNIT = 128, TILE = 64;             // tokens; rows of a stored tile of queries
// Warps that read scores: two groups, which take the two buffers of tensor memory in turn, of eight: a warp has 32 lanes and half of the columns.
constexpr int GROUP = 8, READERS = 2 * GROUP;
constexpr int THREADS = (READERS + 6) * 32, CONVERT = READERS, ISSUE = READERS + 4, FETCH = READERS + 5;
constexpr int CHUNK = TILE * 128;                // bytes of a tile's piece in 64 coordinates
constexpr int IMAGE = 4 * CHUNK;                 // a tile: [2 pieces][2 halves of the coordinates][64 rows][128 bytes], 128-byte swizzle
constexpr int CODES = UNIT * 256;                // a unit's codes in fp16: [2 halves of the coordinates][128 tokens][128 bytes], likewise
constexpr float MOVE = 8.f;
constexpr float TOP = 2047.f * 2048.f;           // a row's largest integer
constexpr unsigned TMEM_COLS = 512;
constexpr unsigned ID = (1u << 4) | ((unsigned)(UNIT >> 3) << 17) | ((unsigned)(UNIT >> 4) << 24);     // 128 x 128, fp16, both K-major

struct MassArgs {
    gbs_kv_attn a;
    KvLine line;
    long long slots;                             // tiles of a KV head: n_tokens * group / 64 + n_items + 2
    unsigned char* rows;                         // [heads][slots][IMAGE]
    float *factor, *lift, *norm;                 // [heads][slots][64]: a row's factor, its sum times that, log2 of its sum of 2^z
    int *lo, *hi;                                // the same: what a row sees
    float2* parts;                               // [blocks][2][128]: m and the sum
    KvJoin* joins;
    // of the second pass: KV heads (a.c.heads counts each of them once for each share of its rows), shares, and what each of these adds up, [shares][n_items][heads][width]
    int heads, shares;
    float* sums;
    const float* base;
    float* mass;
    long long width;
    float decay;
    int* gave_up;                                // [2]: whether a wait ran out in the first pass, in the second: sums that are not whole are not written
    int* status;
};

__device__ __forceinline__ long long slot_of(const MassArgs& P, int head, int item, int first)
{
    return head * P.slots + (((long long)first * P.a.group) >> 6) + item;
}

// byte of a 16-byte piece (8 coordinates) of a row among `N` rows
template <int N>
__device__ __forceinline__ unsigned piece_at(int row, int piece)
{
    return (unsigned)(piece >> 3) * (N * 128) + (unsigned)(row >> 3) * 1024 + (unsigned)(row & 7) * 128 + (unsigned)(((piece & 7) ^ (row & 7)) << 4);
}

// ---- query rows: a warp four heads of a token, eight lanes a row ----
__global__ __launch_bounds__(256) void k_tc_kvmass_prepare(const __grid_constant__ MassArgs P)
{
    kv_wait_before();
    kv_let_next();
    if (blockIdx.x == 0 && threadIdx.x < 2) P.gave_up[threadIdx.x] = 0;
    const gbs_kv_attn& A = P.a;
    const int lane = threadIdx.x & 31, l8 = lane & 7, fours = (A.n_heads + 3) >> 2;
    const long long job = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int token = (int)(job / fours), head = 4 * (int)(job - (long long)token * fours) + (lane >> 3);
    if (token >= A.n_tokens) return;
    const int item = A.cu ? kv_item_of(A.cu, A.n_items, token) : token;
    if (item >= A.n_items) return;
    const KvItem x = kv_item(A, item);
    const int at = token - x.first;
    if (at < 0 || at >= min(x.count, A.max_tokens)) return;
    const bool have = head < A.n_heads;
    float y[16];
    uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (have) {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(A.q) + token * A.q_token + head * A.q_head;
        if (8 * l8 < A.d) raw[0] = *reinterpret_cast<const uint4*>(q + 8 * l8);
        if (64 + 8 * l8 < A.d) raw[1] = *reinterpret_cast<const uint4*>(q + 64 + 8 * l8);
    }
    kv_unpack_bf16(raw[0], y);
    kv_unpack_bf16(raw[1], y + 8);
    kv_hadamard(y, l8);
    float m = 0.f, wrong = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        m = fmaxf(m, fabsf(y[i]));
        wrong += y[i] * 0.f;                     // a row that is not finite has a factor that is not a number
    }
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, h));
        wrong += __shfl_xor_sync(0xffffffffu, wrong, h);
    }
    const float up = m < 1e-28f ? 1.2379400392853803e27f : 1.f;     // 2^90
    const float by = m > 0.f ? TOP / (m * up) : 0.f;
    int q[16], sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        q[i] = __float2int_rn(fminf(fmaxf(y[i] * up * by, -TOP), TOP));
        sum += q[i];
    }
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, h);
    if (!have) return;
    const int kvh = head / A.group, r = at * A.group + (head - kvh * A.group);
    const long long slot = slot_of(P, kvh, item, x.first) + (r >> 6);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __half high[8], low[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int v = q[8 * half + i], h = (v + 1024) >> 11;    // -2047 .. 2047, and what is left -1024 .. 1023
            high[i] = __int2half_rn(h);
            low[i] = __int2half_rn(v - (h << 11));
        }
        unsigned char* to = P.rows + slot * IMAGE + piece_at<TILE>(r & 63, 8 * half + l8);
        // coordinates in the order in which a word of codes gives them
        *reinterpret_cast<uint4*>(to) = make_uint4(as_u(__halves2half2(high[0], high[4])), as_u(__halves2half2(high[1], high[5])),
                                                   as_u(__halves2half2(high[2], high[6])), as_u(__halves2half2(high[3], high[7])));
        *reinterpret_cast<uint4*>(to + 2 * CHUNK) = make_uint4(as_u(__halves2half2(low[0], low[4])), as_u(__halves2half2(low[1], low[5])),
                                                               as_u(__halves2half2(low[2], low[6])), as_u(__halves2half2(low[3], low[7])));
    }
    if (l8 == 0) {
        const float f = m * (A.scale * (KV_NORM * 1.4426950408889634f / TOP)) + wrong;
        P.factor[slot * TILE + (r & 63)] = f;
        P.lift[slot * TILE + (r & 63)] = (float)sum * f;
        KvEntry e = {};
        e.before = x.length - x.count;
        e.length = x.length;
        P.lo[slot * TILE + (r & 63)] = kv_row_lo(A, e, at);
        P.hi[slot * TILE + (r & 63)] = kv_row_hi(A, e, at);
    }
}

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 both(float x) { return pk(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ f32x2 pair(float a, float b) { return pk(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ unsigned uniform(unsigned x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ float no_inf(float x) { return fmaf(x, 0.f, x); }
// a warp's segment becomes the next one
template <int PART = KV_WHOLE>
__device__ __forceinline__ void to_next(const gbs_kv_attn& A, const KvLine& L, KvSeg& seg, int lane)
{
    KvSeg next = seg;
    kv_next<PART>(A, L, next);
    __syncwarp();
    if (lane == 0) seg = next;
    __syncwarp();
}

// 8 columns of this thread's lane of tensor memory; the wait names the registers so that nothing is scheduled across it
__device__ __forceinline__ void tmem_ld8_issue(unsigned taddr, unsigned r[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait8x4(unsigned a[8], unsigned b[8], unsigned c[8], unsigned d[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]),
          "+r"(b[0]), "+r"(b[1]), "+r"(b[2]), "+r"(b[3]), "+r"(b[4]), "+r"(b[5]), "+r"(b[6]), "+r"(b[7]),
          "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]), "+r"(c[4]), "+r"(c[5]), "+r"(c[6]), "+r"(c[7]),
          "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]), "+r"(d[4]), "+r"(d[5]), "+r"(d[6]), "+r"(d[7]) :: "memory");
}
// the warps that read scores meet; whether any of their threads says so
__device__ __forceinline__ bool meet_any(bool x)
{
    int any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((int)x), "n"(READERS * 32) : "memory");
    return any != 0;
}

// A token's key codes and scale, from a page; fetched a unit ahead.
template <bool ASYM>
struct Key {
    uint4 codes[4];
    float scale, low;
    bool there;
    __device__ __forceinline__ void fetch(const gbs_kv_view& c, int page, int head, int pos, bool wanted)
    {
        there = wanted && (unsigned)page < (unsigned)c.n_pages;
        const int ps = 1 << c.page_log, slot = pos & (ps - 1);
        const unsigned char* block = kv_block(c, there ? page : 0, head);
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[i] = reinterpret_cast<const uint4*>(block + slot * KV_ROW)[i];
        const float* s = reinterpret_cast<const float*>(block + 2 * ps * KV_ROW);
        scale = ASYM ? s[2 * slot] : s[slot];
        low = ASYM ? s[2 * slot + 1] : 0.f;
    }
    // codes into row `row` of a unit's tile
    __device__ __forceinline__ void store(unsigned char* tile, int row) const
    {
        const unsigned first = smem_u32(tile) + piece_at<UNIT>(row, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint4 q = codes[i >> 2];
            unsigned c[4];
            kv_codes_f16<ASYM>((i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w, c);
            st_shared_v4((first ^ (unsigned)((i & 7) << 4)) + (i >> 3) * (UNIT * 128), make_uint4(c[0], c[1], c[2], c[3]));
        }
    }
    // what its scores are multiplied by: not a number where the scale is not finite; 0 where the token is not there
    __device__ __forceinline__ float by() const { return there ? no_inf(fmaf(low, 0.f, scale)) : 0.f; }
    __device__ __forceinline__ float middle() const { return there && ASYM ? fmaf(8.f, scale, low) : 0.f; }
};

// 128 rows of A times 128 rows of B, over 128 coordinates
__device__ __forceinline__ void product(unsigned d, unsigned a_lo, unsigned b_lo, unsigned hi)
{
    umma_f16_words<false>(d, a_lo, hi, b_lo, hi, ID);
#pragma unroll
    for (int k = 1; k < 8; ++k) {                // sixteen coordinates: 32 bytes, four of them in a block of 64
        const unsigned step = (k & 3) ? 2u : (unsigned)((UNIT * 128 - 96) >> 4);
        a_lo += step;
        b_lo += step;
        umma_f16_words<true>(d, a_lo, hi, b_lo, hi, ID);
    }
}

// log2 of a row's sum of 2^z, from m and the sum of 2^(z - m): one float, so that all of a row's weights are off by up to 2^-24 of it, which is also what a score is off by.  (m and 1 / sum apart,
// or a factor for what the float leaves out: 47 -> 51 us and 141 -> 151, since a thread has 80 registers, whichever rows they are kept for.)  From 2^24 on floats have no units, and m, added up, may
// be a few of its last bits below the largest score: there the norm is put above that, so that weights are finite.
__device__ __forceinline__ float norm_of(float m, float sum)
{
    const float norm = m + log2f(sum);
    return sum == 0.f ? INFINITY : fabsf(norm) < 16777216.f ? norm : fmaf(fabsf(norm), 4.76837158203125e-7f, norm);      // 2^-21
}

// ---------------------------------------------------------------------------------------------
// first pass
// ---------------------------------------------------------------------------------------------
struct RowsSmem {
    unsigned char q[2][UNIT * 256];              // upper and lower pieces of 128 rows
    unsigned char k[2][CODES];                   // unit i in [i & 1]
    float by[4][UNIT], middle[4][UNIT];          // of unit i in [i & 3]: a unit's scores are read before the one four further is converted
    unsigned there[4][4];
    float2 part[4][UNIT];
    unsigned long long qfull, qfree, kfull[2], kfree[2], dfull[2], dfree[2], drain;
    KvSeg seg, own[THREADS / 32];                // the block's first segment; each warp's present one (in registers it would be spilled, and fetched from L2)
    long long share[THREADS / 32];
    unsigned tmem;
    int abort;
};
static_assert(sizeof(RowsSmem) + 1024 <= 227 * 1024, "one block of an SM");

template <bool ASYM, bool TEST>
__global__ __launch_bounds__(THREADS, 1) void k_tc_kvmass_rows(const __grid_constant__ MassArgs P)
{
    extern __shared__ unsigned char smem_raw[];
    RowsSmem& S = *reinterpret_cast<RowsSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = warp_index();
    if (tid == 0) {
        S.abort = 0;
        mbar_init(&S.qfull, 1);
        mbar_init(&S.qfree, 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(&S.kfull[b], 4);
            mbar_init(&S.kfree[b], 1);
            mbar_init(&S.dfull[b], 2);           // the MMAs, and the thread that has seen the tokens' numbers
            mbar_init(&S.dfree[b], GROUP);
        }
        mbar_init(&S.drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == ISSUE) tmem_alloc(&S.tmem, TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = S.tmem;
    kv_wait_before();
    kv_let_next();
    const int places = kv_share<THREADS>(A, P.line, &S.seg, S.share);
    if (tid == 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};

    KvSeg& seg = S.own[w];
    if (lane == 0) seg = S.seg;
    __syncwarp();
    bool ok = true;
    unsigned it = 0, round = 0, sent = 0;        // units and segments so far, and segments whose rows have been sent for
    for (bool more = places > 0; more && ok;) {
        const KvPiece piece = kv_piece(P.line, seg, places);
        const int n = piece.n, tok0 = ((seg.e.lo >> 7) + piece.skip) * UNIT;
        if (n <= 0) break;                       // the block's last places are in front of a segment's units
        const int item = P.line.by_tiles(seg.index);
        const long long slot = slot_of(P, seg.head, item, seg.e.first) + (seg.e.row0 >> 6);

        if (w < READERS) {
            constexpr int EACH = UNIT / 2;       // tokens of a unit
            const int row = 32 * (w & 3) + lane, half = (w >> 2) & 1, group = w / GROUP, r = seg.e.row0 + row;
            const unsigned at = tmem + ((unsigned)(32 * (w & 3)) << 16) + 256 * group + EACH * half;
            const bool have = r < seg.e.rows;
            const float f = have ? P.factor[slot * TILE + row] : 0.f, lift = have && ASYM ? P.lift[slot * TILE + row] : 0.f;
            const int token = A.by_group(min(r, seg.e.rows - 1));
            const int see_lo = kv_row_lo(A, seg.e, token), see_hi = have ? kv_row_hi(A, seg.e, token) : 0;
            const int all_lo = kv_row_lo(A, seg.e, A.by_group(min(seg.e.rows, seg.e.row0 + UNIT) - 1)), all_hi = kv_row_hi(A, seg.e, A.by_group(seg.e.row0));
            float m = 0.f;
            bool fresh = true;                   // m is none yet
            f32x2 l = both(0.f);
            for (int i = (it + group) & 1; i < n; i += 2) {
                const unsigned now = it + i;
                const int tok = tok0 + i * UNIT + EACH * half;
                if (!(ok = !kv_lost<TEST>(P, &S.abort, 81, round) && mbar_wait_warp(&S.abort, &S.dfull[group], (now >> 1) & 1u, P.status, 81))) break;
                tc_fence_after();
                const uint2 there = *reinterpret_cast<const uint2*>(&S.there[now & 3][2 * half]);
                const bool plain = tok >= all_lo && tok + EACH <= all_hi && (there.x & there.y) == 0xffffffffu;
#pragma unroll 1
                for (int c = 0; c < EACH; c += 16) {
                    unsigned a[16], b[16];
                    tmem_ld16_issue(at + c, a);
                    tmem_ld16_issue(at + 128 + c, b);
                    const float* by = &S.by[now & 3][EACH * half + c];
                    const float* middle = &S.middle[now & 3][EACH * half + c];
                    tmem_ld_wait16x2(a, b);
                    const f32x2 f2 = both(f), lift2 = both(lift), base = both(-m);
                    float z[16];
                    float top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const float4 s = *reinterpret_cast<const float4*>(by + j);
                        f32x2 x0 = fma2(pk(a[j], a[j + 1]), both(2048.f), pk(b[j], b[j + 1])), x1 = fma2(pk(a[j + 2], a[j + 3]), both(2048.f), pk(b[j + 2], b[j + 3]));
                        f32x2 y0 = base, y1 = base;
                        if (ASYM) {
                            const float4 mid = *reinterpret_cast<const float4*>(middle + j);
                            y0 = fma2(pair(mid.x, mid.y), lift2, base);
                            y1 = fma2(pair(mid.z, mid.w), lift2, base);
                        }
                        x0 = fma2(x0, mul2(pair(s.x, s.y), f2), y0);
                        x1 = fma2(x1, mul2(pair(s.z, s.w), f2), y1);
                        unsigned u0, u1, u2, u3;
                        unpk(x0, u0, u1);
                        unpk(x1, u2, u3);
                        z[j] = __uint_as_float(u0); z[j + 1] = __uint_as_float(u1); z[j + 2] = __uint_as_float(u2); z[j + 3] = __uint_as_float(u3);
                    }
                    if (!plain) {
                        const int lo = see_lo - tok - c, hi = see_hi - tok - c;
                        const unsigned which = (c < 32 ? there.x : there.y) >> (c & 31);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (j < lo || j >= hi || !(which >> j & 1)) z[j] = -INFINITY;
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 2) top = max3(z[j], z[j + 1], top);
                    if (top > MOVE || (fresh && top > -INFINITY)) {      // what has been added up changes by an exact power of two
                        const float step = ceilf(top);
                        if (!fresh) l = mul2(l, both(kv_ex2(-step)));    // (before, it is 0, or a NaN that stays)
                        m += step;
                        fresh = false;
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] -= step;
                    }
                    f32x2 l2[2] = {both(0.f), both(0.f)};
#pragma unroll
                    for (int j = 0; j < 16; j += 2) l2[(j >> 1) & 1] = add2(l2[(j >> 1) & 1], pair(kv_ex2(z[j]), kv_ex2(z[j + 1])));
                    l = add2(l, add2(l2[0], l2[1]));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.dfree[group]);
            }
            unsigned u0, u1;
            unpk(l, u0, u1);
            const float sum = __uint_as_float(u0) + __uint_as_float(u1), top = fresh ? NONE : m;
            S.part[2 * group + half][row] = make_float2(top, sum);
            if (meet_any(!ok)) { ok = false; break; }
            if (w < 4 && have) {
                float whole = NONE, total = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) whole = fmaxf(whole, S.part[x][row].x);
#pragma unroll
                for (int x = 0; x < 4; ++x) total += S.part[x][row].y * kv_ex2(S.part[x][row].x - whole);
                if (piece.starts && piece.ends) P.norm[slot * TILE + row] = norm_of(whole, total);
                else P.parts[((long long)blockIdx.x * 2 + (piece.starts ? 1 : 0)) * UNIT + row] = make_float2(whole, total);
            }
            if (tid == 0 && piece.starts && !piece.ends) P.joins[blockIdx.x] = kv_join(P.line, seg, places);
            meet_any(false);                     // the parts have been read
        } else if (w < ISSUE) {
            const int me = tid - CONVERT * 32;
            const int* pages = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            const auto page_of = [&](int tok) { return tok < seg.e.hi ? pages[tok >> A.c.page_log] : -1; };
            const auto wanted = [&](int tok) { return tok >= seg.e.lo && tok < seg.e.hi; };
            Key<ASYM> key;                       // a unit ahead (two: no faster)
            key.fetch(A.c, page_of(tok0 + me), seg.head, tok0 + me, wanted(tok0 + me));
            int page = page_of(tok0 + UNIT + me);
            for (int i = 0; i < n; ++i) {
                const unsigned now = it + i;
                const int b = now & 1;
                if (now > 1 && !(ok = !kv_lost<TEST>(P, &S.abort, 82, round) && mbar_wait_warp(&S.abort, &S.kfree[b], ((now >> 1) + 1) & 1u, P.status, 82))) break;
                key.store(S.k[b], me);
                S.by[now & 3][me] = key.by();
                if (ASYM) S.middle[now & 3][me] = key.middle();
                const unsigned there = __ballot_sync(0xffffffffu, key.there);
                if (lane == 0) S.there[now & 3][w - CONVERT] = there;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.kfull[b]);
                if (i + 1 < n) {
                    const int next = tok0 + (i + 1) * UNIT + me;
                    key.fetch(A.c, page, seg.head, next, wanted(next));
                    page = page_of(next + UNIT);
                }
            }
        } else if (w == ISSUE) {
            const unsigned long long qd = smem_desc(smem_u32(S.q[0]), 16, 1024, 2), kd = smem_desc(smem_u32(S.k[0]), 16, 1024, 2);
            const unsigned q_lo = (unsigned)qd, k_lo = (unsigned)kd, hi = (unsigned)(qd >> 32), to = uniform(tmem), at0 = uniform(it);
            const int units = (int)uniform((unsigned)n);
            ok = !kv_lost<TEST>(P, &S.abort, 83, round) && mbar_wait_warp(&S.abort, &S.qfull, uniform(round) & 1u, P.status, 83);
            for (int i = 0; i < units && ok; ++i) {
                const unsigned now = at0 + i, b = now & 1;
                if (!(ok = !kv_lost<TEST>(P, &S.abort, 84, round) && mbar_wait_warp(&S.abort, &S.kfull[b], (now >> 1) & 1u, P.status, 84))) break;
                if (now > 1 && !(ok = !kv_lost<TEST>(P, &S.abort, 85, round) && mbar_wait_warp(&S.abort, &S.dfree[b], ((now >> 1) + 1) & 1u, P.status, 85))) break;
                tc_fence_after();
                product(to + 256 * b, q_lo, k_lo + b * (CODES >> 4), hi);
                product(to + 256 * b + 128, q_lo + (UNIT * 256 >> 4), k_lo + b * (CODES >> 4), hi);
                umma_commit(&S.kfree[b]);
                umma_commit(&S.dfull[b]);
                if (lane == 0) mbar_arrive(&S.dfull[b]);
            }
            if (ok) umma_commit(&S.qfree);
        } else {
            if (round > 0) ok = !kv_lost<TEST>(P, &S.abort, 86, round) && mbar_wait_warp(&S.abort, &S.qfree, (round - 1) & 1u, P.status, 86);
            if (ok) ++sent;
            if (ok && lane == 0) {
                mbar_arrive_expect_tx(&S.qfull, 2 * IMAGE);
#pragma unroll
                for (int x = 0; x < 8; ++x) {    // tile, piece, half of the coordinates
                    const int tile = x >> 2, part = (x >> 1) & 1, kb = x & 1;
                    bulk_load(S.q[part] + kb * (UNIT * 128) + tile * CHUNK, P.rows + (slot + tile) * IMAGE + (2 * part + kb) * CHUNK, CHUNK, &S.qfull);
                }
            }
            __syncwarp();
        }
        if (!ok) break;
        it += n;
        ++round;
        more = kv_more(P.line, seg, places);
        if (more) to_next(A, P.line, seg, lane);
    }
    tc_fence_before();
    __syncthreads();
    if (S.abort) {                               // a wait has run out: what is under way is given time to end
        if (tid == 0) P.gave_up[0] = 1;
        if (w == ISSUE) {
            umma_commit(&S.drain);
            drain_copies(&S.drain, 1, 1);
        }
        if (w == FETCH) drain_copies(&S.qfull, 1, (int)sent);
    }
    if (w == ISSUE) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

// The sums of rows whose segments several blocks share: block b joins the one that starts in block b.
__global__ __launch_bounds__(UNIT) void k_tc_kvmass_join(const __grid_constant__ MassArgs P)
{
    kv_wait_before();
    kv_let_next();
    const KvJoin j = P.joins[blockIdx.x];
    if (j.blocks == 0) return;
    const KvEntry e = kv_entry(P.a, P.line, j.index);
    if (e.row0 + (int)threadIdx.x >= e.rows) return;
    const float2* first = P.parts + ((long long)blockIdx.x * 2 + 1) * UNIT + threadIdx.x;
    float top = NONE, sum = 0.f;
    for (int b = 0; b < j.blocks; ++b) {
        const float2 x = *(b == 0 ? first : first + (long long)(2 * b - 1) * UNIT);
        const float now = fmaxf(top, x.x);
        sum = sum * kv_ex2(top - now) + x.y * kv_ex2(x.x - now);
        top = now;
    }
    P.norm[(slot_of(P, j.head, P.line.by_tiles(j.index), e.first) + (e.row0 >> 6)) * TILE + threadIdx.x] = norm_of(top, sum);
}

// ---------------------------------------------------------------------------------------------
// second pass
// ---------------------------------------------------------------------------------------------
// Where no item has more than two tiles of rows (STAY), they stay in shared memory for all of a segment's pairs of units, and a pair's codes are converted while the one
// before is worked on.  With more, tiles pass through a ring of four for each pair: a fetch takes as long as two or three of them are worked on.
template <bool STAY>
struct TokensSmem {
    static constexpr int PAIRS = STAY ? 2 : 1, TILES = STAY ? 2 : 4;
    unsigned char k[PAIRS][2][CODES];            // pair p in [p % PAIRS]
    unsigned char q[TILES][IMAGE];               // [2 halves of the coordinates][upper pieces of 64 rows, lower pieces][128 bytes]
    float factor[TILES][TILE], lift[TILES][TILE], norm[TILES][TILE];
    int lo[TILES][TILE], hi[TILES][TILE];
    float by[PAIRS][2 * UNIT], middle[PAIRS][2 * UNIT];
    unsigned there[PAIRS][8];
    float part[2][4][2 * UNIT];
    unsigned long long qfull[TILES], qfree[TILES], kfull[PAIRS], kfree[PAIRS], dfull[2], dfree[2], drain;
    KvSeg seg, own[THREADS / 32];                // the block's first segment; each warp's present one (in registers it would be spilled, and fetched from L2)
    long long share[THREADS / 32];
    unsigned tmem;
    int abort;
};
static_assert(sizeof(TokensSmem<true>) + 1024 <= 227 * 1024 && sizeof(TokensSmem<false>) + 1024 <= 227 * 1024, "one block of an SM");

template <bool ASYM, bool STAY, bool TEST>
__global__ __launch_bounds__(THREADS, 1) void k_tc_kvmass_tokens(const __grid_constant__ MassArgs P)
{
    extern __shared__ unsigned char smem_raw[];
    using Smem = TokensSmem<STAY>;
    constexpr unsigned PAIRS = Smem::PAIRS, TILES = Smem::TILES;
    Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = warp_index();
    if (tid == 0) {
        S.abort = 0;
        for (int b = 0; b < (int)TILES; ++b) {
            mbar_init(&S.qfull[b], 1);
            mbar_init(&S.qfree[b], 1 + (STAY ? READERS : GROUP));
        }
        for (int b = 0; b < (int)PAIRS; ++b) {
            mbar_init(&S.kfull[b], 4);
            mbar_init(&S.kfree[b], 1 + READERS);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&S.dfull[b], 1);
            mbar_init(&S.dfree[b], GROUP);
        }
        mbar_init(&S.drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == ISSUE) tmem_alloc(&S.tmem, TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = S.tmem;
    kv_wait_before();
    kv_let_next();
    // without all rows' sums the weights stay what they are
    const bool lost = P.gave_up[0] != 0;
    int places = kv_share<THREADS, KV_ALL>(A, P.line, &S.seg, S.share);
    if (lost) places = 0;

    KvSeg& seg = S.own[w];
    if (lane == 0) seg = S.seg;
    __syncwarp();
    bool ok = true;
    unsigned pp = 0, dt = 0, round = 0;          // pairs, (pair, tile)s and segments so far
    // STAY: segments so far, each of which fills a buffer for each of its tiles once, or the second buffer's fillings; else fillings of the ring.  Three roles keep count.
    unsigned used = 0, used1 = 0;
    unsigned sent = 0, sent1 = 0;                // STAY: fillings of the two buffers that have been sent for: a segment's begin before, or after, another role gives up
    for (bool more = places > 0; more && ok;) {
        const KvPiece piece = kv_piece(P.line, seg, places);
        if (piece.n <= 0) break;
        const int tok0 = piece.skip * 2 * UNIT;  // the line counts pairs of units here; the last pair of a sequence may be one unit
        const int n = min(2 * piece.n, max(1, (seg.e.length - tok0 + UNIT - 1) / UNIT));
        // the tiles that are this segment's share: every `stride`-th of them from `part` on
        const int stride = STAY ? 1 : P.shares, head = STAY ? seg.head : seg.head / stride, part = STAY ? 0 : seg.head - head * stride;
        const long long slot = slot_of(P, head, seg.index, seg.e.first);
        const int pairs = (n + 1) >> 1, tiles = (seg.e.rows + TILE - 1) / TILE;
        // whether any row of a tile sees any token of a pair; whether all of its 64 rows see all of them
        const auto sees = [&](int pair, int tile) {
            const int a = tok0 + 2 * UNIT * pair, last = min(seg.e.rows, TILE * (tile + 1)) - 1;
            return a < kv_row_hi(A, seg.e, A.by_group(last)) && a + 2 * UNIT > kv_row_lo(A, seg.e, A.by_group(TILE * tile));
        };
        const auto all = [&](int pair, int tile) {
            const int a = tok0 + 2 * UNIT * pair;
            return TILE * (tile + 1) <= seg.e.rows && a >= kv_row_lo(A, seg.e, A.by_group(TILE * (tile + 1) - 1)) && a + 2 * UNIT <= kv_row_hi(A, seg.e, A.by_group(TILE * tile));
        };

        if (w < READERS) {
            constexpr int EACH = TILE / 2;       // rows of a tile
            const int half = (w >> 2) & 1, group = w / GROUP, me = 32 * (w & 3) + lane;
            const unsigned at = tmem + ((unsigned)(32 * (w & 3)) << 16) + 256 * group + EACH * half;
            for (int p = 0; p < pairs; ++p) {
                const unsigned now = pp + p, kb = now % PAIRS;
                const int units = min(2, n - 2 * p);
                float acc[2] = {0.f, 0.f}, off[2] = {0.f, 0.f};      // sums over many rows, with what their rounding has left out
                if (ok) ok = !kv_lost<TEST>(P, &S.abort, 91, round) && mbar_wait_warp(&S.abort, &S.kfull[kb], (now / PAIRS) & 1u, P.status, 91);
                const float by0 = S.by[kb][me], by1 = S.by[kb][UNIT + me], mid0 = ASYM ? S.middle[kb][me] : 0.f, mid1 = ASYM ? S.middle[kb][UNIT + me] : 0.f;
                const bool all_there = (S.there[kb][w & 3] & (units > 1 ? S.there[kb][4 + (w & 3)] : 0xffffffffu)) == 0xffffffffu;
                const bool there0 = S.there[kb][w & 3] >> lane & 1, there1 = units > 1 && (S.there[kb][4 + (w & 3)] >> lane & 1);
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.kfree[kb]);
                for (int tile = part; tile < tiles && ok; tile += stride) {
                    if (!sees(p, tile)) continue;
                    const unsigned b = STAY ? tile : used % TILES, filled = STAY ? (tile ? used1 : used) : used / TILES;     // fillings of the buffer before this one
                    if (!STAY) ++used;
                    if ((dt++ & 1) != (unsigned)group) continue;
                    const unsigned turn = (dt - 1) >> 1;
                    if (!(ok = !kv_lost<TEST>(P, &S.abort, 92, round) && mbar_wait_warp(&S.abort, &S.qfull[b], filled & 1u, P.status, 92))) break;
                    if (!(ok = !kv_lost<TEST>(P, &S.abort, 93, round) && mbar_wait_warp(&S.abort, &S.dfull[group], turn & 1u, P.status, 93))) break;
                    tc_fence_after();
                    const bool plain = all_there && all(p, tile);    // what is taken for a second unit that there is not goes nowhere
                    f32x2 got0 = both(0.f), got1 = both(0.f);
#pragma unroll 1
                    for (int c = 0; c < EACH; c += 8) {
                        const unsigned from = at + c;
                        unsigned a0[8], b0[8], a1[8], b1[8];
                        tmem_ld8_issue(from, a0);
                        tmem_ld8_issue(from + 64, b0);
                        tmem_ld8_issue(from + 128, a1);
                        tmem_ld8_issue(from + 192, b1);
                        tmem_ld_wait8x4(a0, b0, a1, b1);
                        const int r0 = EACH * half + c;
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const float4 f4 = *reinterpret_cast<const float4*>(&S.factor[b][r0 + j]), c4 = *reinterpret_cast<const float4*>(&S.norm[b][r0 + j]);
                            const float4 l4 = ASYM ? *reinterpret_cast<const float4*>(&S.lift[b][r0 + j]) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int k = j + 2 * h;
                                const f32x2 f2 = h ? pair(f4.z, f4.w) : pair(f4.x, f4.y), c2 = h ? pair(-c4.z, -c4.w) : pair(-c4.x, -c4.y);
                                const f32x2 l2 = h ? pair(l4.z, l4.w) : pair(l4.x, l4.y);
                                f32x2 x0 = fma2(pk(a0[k], a0[k + 1]), both(2048.f), pk(b0[k], b0[k + 1])), x1 = fma2(pk(a1[k], a1[k + 1]), both(2048.f), pk(b1[k], b1[k + 1]));
                                x0 = fma2(x0, mul2(both(by0), f2), ASYM ? fma2(both(mid0), l2, c2) : c2);
                                x1 = fma2(x1, mul2(both(by1), f2), ASYM ? fma2(both(mid1), l2, c2) : c2);
                                unsigned u[4];
                                unpk(x0, u[0], u[1]);
                                unpk(x1, u[2], u[3]);
                                float e[4];
#pragma unroll
                                for (int x = 0; x < 4; ++x) e[x] = kv_ex2(__uint_as_float(u[x]));
                                if (!plain) {
                                    const int2 lo = *reinterpret_cast<const int2*>(&S.lo[b][r0 + k]), hi = *reinterpret_cast<const int2*>(&S.hi[b][r0 + k]);
#pragma unroll
                                    for (int x = 0; x < 4; ++x) {
                                        const int pos = tok0 + 2 * UNIT * p + (x >> 1) * UNIT + me;
                                        if (TILE * tile + r0 + k + (x & 1) >= seg.e.rows || pos < (x & 1 ? lo.y : lo.x) || pos >= (x & 1 ? hi.y : hi.x) || !(x >> 1 ? there1 : there0)) e[x] = 0.f;
                                    }
                                }
                                got0 = add2(got0, pair(e[0], e[1]));
                                got1 = add2(got1, pair(e[2], e[3]));
                            }
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&S.dfree[group]);
                        if (!STAY) mbar_arrive(&S.qfree[b]);
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        unsigned u0, u1;
                        unpk(x ? got1 : got0, u0, u1);
                        const float y = __fsub_rn(__fadd_rn(__uint_as_float(u0), __uint_as_float(u1)), off[x]), sum = __fadd_rn(acc[x], y);
                        off[x] = __fsub_rn(__fsub_rn(sum, acc[x]), y);
                        acc[x] = sum;
                    }
                }
                S.part[now & 1][2 * group + half][me] = acc[0];
                S.part[now & 1][2 * group + half][UNIT + me] = acc[1];
                if (meet_any(!ok)) { ok = false; break; }
                if (group == 0) {
                    const int pos = tok0 + 2 * UNIT * p + half * UNIT + me;
                    if (half < units && pos < seg.e.length && pos < P.width) {
                        float sum = 0.f;
#pragma unroll
                        for (int x = 0; x < 4; ++x) sum += S.part[now & 1][x][half * UNIT + me];
                        const long long to = ((long long)seg.e.seq * P.heads + head) * P.width + pos;
                        if (!STAY && stride > 1) P.sums[(((long long)part * A.n_items + seg.index) * P.heads + head) * P.width + pos] = sum;
                        else P.mass[to] = pos < seg.e.before && P.decay != 0.f ? fmaf(P.decay, P.base[to], sum) : sum;
                    }
                }
            }
            if (STAY && ok) {
                __syncwarp();
                if (lane == 0)
                    for (int b = 0; b < tiles; ++b) mbar_arrive(&S.qfree[b]);
            }
        } else if (w < ISSUE) {
            const int me = tid - CONVERT * 32;
            const int* pages = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
            const auto page_of = [&](int tok) { return tok < seg.e.length ? pages[tok >> A.c.page_log] : -1; };
            Key<ASYM> key;
            key.fetch(A.c, page_of(tok0 + me), head, tok0 + me, tok0 + me < seg.e.length);
            int page = page_of(tok0 + UNIT + me);
            for (int i = 0; i < n; ++i) {
                const unsigned now = pp + (i >> 1), kb = now % PAIRS;
                if ((i & 1) == 0 && now >= PAIRS && !(ok = !kv_lost<TEST>(P, &S.abort, 94, round) && mbar_wait_warp(&S.abort, &S.kfree[kb], (now / PAIRS + 1) & 1u, P.status, 94))) break;
                key.store(S.k[kb][i & 1], me);
                S.by[kb][(i & 1) * UNIT + me] = key.by();
                if (ASYM) S.middle[kb][(i & 1) * UNIT + me] = key.middle();
                const unsigned there = __ballot_sync(0xffffffffu, key.there);
                if (lane == 0) S.there[kb][4 * (i & 1) + w - CONVERT] = there;
                if ((i & 1) || i + 1 == n) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&S.kfull[kb]);
                }
                if (i + 1 < n) {
                    const int next = tok0 + (i + 1) * UNIT + me;
                    key.fetch(A.c, page, head, next, next < seg.e.length);
                    page = page_of(next + UNIT);
                }
            }
        } else if (w == ISSUE) {
            const unsigned long long qd = smem_desc(smem_u32(S.q[0]), 16, 1024, 2), kd = smem_desc(smem_u32(S.k[0][0]), 16, 1024, 2);
            const unsigned q_lo = (unsigned)qd, k_lo = (unsigned)kd, hi = (unsigned)(qd >> 32), to = uniform(tmem);
            const int all_units = (int)uniform((unsigned)n), all_pairs = (int)uniform((unsigned)pairs), all_tiles = (int)uniform((unsigned)tiles);
            for (int p = 0; p < all_pairs && ok; ++p) {
                const unsigned now = uniform(pp) + p, kb = now % PAIRS;
                if (!(ok = !kv_lost<TEST>(P, &S.abort, 95, round) && mbar_wait_warp(&S.abort, &S.kfull[kb], (now / PAIRS) & 1u, P.status, 95))) break;
                for (int tile = (int)uniform(part); tile < all_tiles; tile += (int)uniform(stride)) {
                    if (!uniform(sees(p, tile))) continue;
                    const unsigned u = uniform(used), u1 = uniform(used1), b = STAY ? tile : u % TILES, filled = STAY ? (tile ? u1 : u) : u / TILES, d = uniform(dt);
                    if (!(ok = !kv_lost<TEST>(P, &S.abort, 96, round) && mbar_wait_warp(&S.abort, &S.qfull[b], filled & 1u, P.status, 96))) break;
                    if (d > 1 && !(ok = !kv_lost<TEST>(P, &S.abort, 97, round) && mbar_wait_warp(&S.abort, &S.dfree[d & 1], ((d >> 1) + 1) & 1u, P.status, 97))) break;
                    tc_fence_after();
                    product(to + 256 * (d & 1), k_lo + 2 * kb * (CODES >> 4), q_lo + b * (IMAGE >> 4), hi);
                    if (2 * p + 1 < all_units) product(to + 256 * (d & 1) + 128, k_lo + (2 * kb + 1) * (CODES >> 4), q_lo + b * (IMAGE >> 4), hi);
                    umma_commit(&S.dfull[d & 1]);
                    if (!STAY) umma_commit(&S.qfree[b]);
                    ++dt;
                    if (!STAY) ++used;
                }
                if (ok) umma_commit(&S.kfree[kb]);
            }
            if (STAY)                            // a tile that no token of the segment is seen by has come all the same
                for (int b = 0; b < all_tiles && ok; ++b) {
                    ok = !kv_lost<TEST>(P, &S.abort, 99, round) && mbar_wait_warp(&S.abort, &S.qfull[b], uniform(b ? used1 : used) & 1u, P.status, 99);
                    if (ok) umma_commit(&S.qfree[b]);
                }
        } else {
            const auto fill = [&](int tile, unsigned b, unsigned filled) {
                if (filled > 0 && (kv_lost<TEST>(P, &S.abort, 98, round) || !mbar_wait_warp(&S.abort, &S.qfree[b], (filled - 1) & 1u, P.status, 98))) return false;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&S.qfull[b], IMAGE + 5 * TILE * 4);
#pragma unroll
                    for (int x = 0; x < 4; ++x)  // piece, half of the coordinates
                        bulk_load(S.q[b] + (x & 1) * (UNIT * 128) + (x >> 1) * CHUNK, P.rows + (slot + tile) * IMAGE + x * CHUNK, CHUNK, &S.qfull[b]);
                    bulk_load(S.factor[b], P.factor + (slot + tile) * TILE, TILE * 4, &S.qfull[b]);
                    bulk_load(S.lift[b], P.lift + (slot + tile) * TILE, TILE * 4, &S.qfull[b]);
                    bulk_load(S.norm[b], P.norm + (slot + tile) * TILE, TILE * 4, &S.qfull[b]);
                    bulk_load(S.lo[b], P.lo + (slot + tile) * TILE, TILE * 4, &S.qfull[b]);
                    bulk_load(S.hi[b], P.hi + (slot + tile) * TILE, TILE * 4, &S.qfull[b]);
                }
                __syncwarp();
                return true;
            };
            if (STAY) {
                for (int tile = 0; tile < tiles && ok; ++tile) {
                    ok = fill(tile, tile, tile ? used1 : used);
                    if (ok) ++(tile ? sent1 : sent);
                }
            } else {
                for (int p = 0; p < pairs && ok; ++p)
                    for (int tile = part; tile < tiles && ok; tile += stride)
                        if (sees(p, tile) && (ok = fill(tile, used % TILES, used / TILES))) ++used;
            }
        }
        if (!ok) break;
        pp += pairs;
        ++round;
        if (STAY) {
            ++used;
            if (tiles > 1) ++used1;
        }
        more = kv_more(P.line, seg, places);
        if (more) to_next<KV_ALL>(A, P.line, seg, lane);
    }
    tc_fence_before();
    __syncthreads();
    if (S.abort) {
        if (tid == 0) P.gave_up[1] = 1;
        if (w == ISSUE) {
            umma_commit(&S.drain);
            drain_copies(&S.drain, 1, 1);
        }
        if (w == FETCH) {                           // the copies that were sent for last.  (A wait for one that was not would pass at once: it goes by its parity)
            if (STAY) {
                drain_copies(&S.qfull[0], 1, (int)sent);
                drain_copies(&S.qfull[1], 1, (int)sent1);
            } else {
                drain_copies(S.qfull, TILES, (int)used);
            }
        }
    }
    if (w == ISSUE) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

// What the shares of a KV head's rows have added up.
__global__ __launch_bounds__(256) void k_tc_kvmass_sums(const __grid_constant__ MassArgs P)
{
    kv_wait_before();
    kv_let_next();
    const gbs_kv_attn& A = P.a;
    const int item = blockIdx.x / P.heads, head = blockIdx.x - item * P.heads;
    const KvEntry e = kv_entry<KV_ALL>(A, P.line, item);
    if (e.units == 0 || P.gave_up[0] || P.gave_up[1]) return;
    const long long row = ((long long)e.seq * P.heads + head) * P.width, step = (long long)A.n_items * P.heads * P.width;
    const float* sums = P.sums + ((long long)item * P.heads + head) * P.width;
    for (long long pos = 256ll * blockIdx.y + threadIdx.x; pos < e.length && pos < P.width; pos += 256ll * gridDim.y) {
        float sum = 0.f;
        for (int i = 0; i < P.shares; ++i) sum += sums[i * step + pos];
        P.mass[row + pos] = pos < e.before && P.decay != 0.f ? fmaf(P.decay, P.base[row + pos], sum) : sum;
    }
}

int64_t round_up(int64_t x) { return (x + 15) & ~(int64_t)15; }
// In the second pass a block has a pair of units and all rows that see them, of which a few thousand tokens have too few to go round (6000 tokens, 4 KV heads: 96 pairs for 148 SMs).  So the
// tiles of rows are shared among segments where that is likely to be done sooner, by the pairs that the width has: the most that a block has to do counts, and a segment's start takes as long as one
// and a half tiles.  1000 tokens of 4 query heads a KV head: 94 us undivided, 69 in three shares, 85 in eight.  The shares' sums need room by the width.
constexpr int MOST_SHARES = 8;
constexpr int64_t MOST_SUMS = 64ll << 20;
int shares_of(const gbs_plan* p, const gbs_kv_attn& A, int64_t width)
{
    const int64_t tiles = ((int64_t)std::min<int64_t>(A.max_tokens, A.n_tokens) * A.group + TILE - 1) / TILE, segments = (int64_t)A.n_items * A.c.heads;
    const int64_t pairs = std::min<int64_t>(width, (int64_t)A.c.max_pages << A.c.page_log) / (2 * UNIT) + 1;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= MOST_SHARES && (s == 1 || 4 * s <= tiles); ++s) {
        if (s > 1 && (segments == 0 || width > MOST_SUMS / (segments * s * (int64_t)sizeof(float)))) break;
        const double cost = (double)((segments * pairs * s + p->sm_count - 1) / p->sm_count) * ((double)tiles / s + 1.5);
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

struct Layout {
    int64_t slots, rows, factor, lift, norm, lo, hi, parts, joins, gave_up, sums, bytes;
};
Layout layout_of(const gbs_plan* p, const gbs_kv_attn& A, int64_t width)
{
    Layout l;
    l.slots = A.n_tokens * A.group / TILE + A.n_items + 2;
    const int64_t all = A.c.heads * l.slots;
    l.rows = 0;
    l.factor = all * IMAGE;
    l.lift = l.factor + all * TILE * (int64_t)sizeof(float);
    l.norm = l.lift + all * TILE * (int64_t)sizeof(float);
    l.lo = l.norm + all * TILE * (int64_t)sizeof(float);
    l.hi = l.lo + all * TILE * (int64_t)sizeof(int);
    l.parts = l.hi + all * TILE * (int64_t)sizeof(int);
    l.joins = l.parts + (int64_t)p->sm_count * 2 * UNIT * sizeof(float2);
    l.gave_up = l.joins + round_up((int64_t)p->sm_count * sizeof(KvJoin));
    l.sums = l.gave_up + 16;
    const int shares = shares_of(p, A, width);
    l.bytes = l.sums + (shares > 1 ? (int64_t)shares * A.n_items * A.c.heads * width * (int64_t)sizeof(float) : 0);
    return l;
}

template <typename K>
int launch(const gbs_plan* p, K kernel, size_t smem, const MassArgs& P, cudaStream_t stream)
{
    const cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return e != cudaSuccess ? (int)e : gbs_kv_launch(p, kernel, dim3((unsigned)p->sm_count), THREADS, smem, stream, P);
}

}  // namespace

int64_t gbs_tc_kvmass_workspace(const gbs_plan* p, const gbs_kv_attn& A, int64_t width) { return layout_of(p, A, width).bytes; }

int gbs_tc_kvmass_launch(const gbs_plan* p, const gbs_kv_attn& A, const float* base, float decay, float* mass, int64_t width, void* workspace,
                         cudaStream_t stream)
{
    const Layout l = layout_of(p, A, width);
    unsigned char* w = static_cast<unsigned char*>(workspace);
    MassArgs P = {};
    P.a = A;
    P.line.unit_log = 7;
    P.line.tile_rows = UNIT;
    P.line.tiles = (int)(((int64_t)A.max_tokens * A.group + UNIT - 1) / UNIT);
    P.line.by_tiles.set((unsigned)P.line.tiles);
    P.line.entries = A.n_items * P.line.tiles;
    P.line.pad = 2;
    P.line.least = 1;
    P.slots = l.slots;
    P.rows = w + l.rows;
    P.factor = reinterpret_cast<float*>(w + l.factor);
    P.lift = reinterpret_cast<float*>(w + l.lift);
    P.norm = reinterpret_cast<float*>(w + l.norm);
    P.lo = reinterpret_cast<int*>(w + l.lo);
    P.hi = reinterpret_cast<int*>(w + l.hi);
    P.parts = reinterpret_cast<float2*>(w + l.parts);
    P.joins = reinterpret_cast<KvJoin*>(w + l.joins);
    P.gave_up = reinterpret_cast<int*>(w + l.gave_up);
    P.base = base;
    P.mass = mass;
    P.width = width;
    P.decay = decay;
    P.status = p->d_status;
    const int64_t jobs = A.n_tokens * ((A.n_heads + 3) / 4);
    const size_t rows_smem = sizeof(RowsSmem) + 1024;
    const bool stay = (int64_t)A.max_tokens * A.group <= 2 * TILE, test = A.lost_code != 0;
    int rc = gbs_kv_launch(p, k_tc_kvmass_prepare, dim3((unsigned)((jobs + 7) / 8)), 256, 0, stream, P);
    if (rc == 0) rc = launch(p, test ? (p->asym ? k_tc_kvmass_rows<true, true> : k_tc_kvmass_rows<false, true>) : (p->asym ? k_tc_kvmass_rows<true, false> : k_tc_kvmass_rows<false, false>), rows_smem, P, stream);
    if (rc == 0) rc = gbs_kv_launch(p, k_tc_kvmass_join, dim3((unsigned)p->sm_count), UNIT, 0, stream, P);
    P.line.unit_log = 8;
    P.line.tile_rows = 1 << 29;                  // a sequence is one tile from here on
    P.line.tiles = 1;
    P.line.by_tiles.set(1);
    P.line.entries = A.n_items;
    P.line.pad = 0;
    if (rc != 0) return rc;
    const size_t smem = (stay ? sizeof(TokensSmem<true>) : sizeof(TokensSmem<false>)) + 1024;
    const auto f = test ? (p->asym ? (stay ? k_tc_kvmass_tokens<true, true, true> : k_tc_kvmass_tokens<true, false, true>)
                                   : (stay ? k_tc_kvmass_tokens<false, true, true> : k_tc_kvmass_tokens<false, false, true>))
                        : (p->asym ? (stay ? k_tc_kvmass_tokens<true, true, false> : k_tc_kvmass_tokens<true, false, false>)
                                   : (stay ? k_tc_kvmass_tokens<false, true, false> : k_tc_kvmass_tokens<false, false, false>));
    P.heads = A.c.heads;
    P.shares = stay ? 1 : shares_of(p, A, width);
    P.a.c.heads *= P.shares;
    P.sums = reinterpret_cast<float*>(w + l.sums);
    rc = launch(p, f, smem, P, stream);
    if (rc != 0 || P.shares == 1) return rc;
    return gbs_kv_launch(p, k_tc_kvmass_sums, dim3((unsigned)A.n_items * (unsigned)A.c.heads, (unsigned)std::min<int64_t>((width + 255) / 256, 1024)), 256, 0, stream, P);
}
