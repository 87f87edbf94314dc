// The softmax weight that each cached token gets from the queries of a call (gbs_kv_attention_mass), for each KV head:
//     mass[j] = decay base[j] + sum over the item's rows r of 2^(z[r][j] - m[r]) / sum_k 2^(z[r][k] - m[r]),
// z the scores in units of log2, m[r] near their largest.  Rows first become integers, then one pass over the keys finds the rows' sums, and a second one
// the tokens'.
//
// Results are fp32, so scores have to be right to fp32 as well: a query row is an integer of 24 bits per coordinate, in three pieces of 8, and key codes
// enter the matrix unit as they are (16 c, a byte whose upper half is the code), so the sums of products are exact integers; what is rounded is the query row (2^-24 of its largest
// coordinate), the integer when it becomes a float, and the scale.
//
// For up to 32 rows of an item and KV head (gbs_tc_kvmass.cu: more) the first pass leaves the scores, 4 bytes a row, for the second, which then need not read keys. What bounds the first is
// its instructions, 480 for 32 tokens and 8 rows by a warp, at 16 warps an SM that leave 45 % of the issue slots empty: 48 sequences of up to 6000 tokens, 8 KV heads of 4 query heads,
// asymmetric, 23 us (the keys at a copy's rate: 9), and 8 for the second; before that 2.7 for the rows, and 2 where sums of divided sequences are joined.  With the codes brought by bulk copies
// instead of 16 bytes a thread it took one less.  (Where there is no room for the scores the second pass finds them again, 33 us.)
#include <algorithm>

#include "gbs_kv_attn.cuh"

namespace {

constexpr int UNIT = 128, THREADS = 128, WARPS = THREADS / 32, STAGES = 3;
constexpr int TILE = 8, PIECES = 3, TILE_BYTES = PIECES * 1024;      // rows that one product takes, and their integers
constexpr int BLOCKS_PER_SM = 4;             // of one tile at a time (us, 48 sequences): 2: 32, 3: 23.9, 4: 23.2, 5: 24.2, 6: 27.4
constexpr float MOVE = 8.f;                                          // a maximum moves when a score is so much (log2) above it
constexpr float TOP = 127.f * 65536.f;                               // a row's largest integer
static_assert(UNIT == WARPS * 32, "a warp has 32 tokens of a unit");

struct MassArgs {
    gbs_kv_attn a;
    KvLine line;
    long long tiles;                             // of a KV head: n_tokens * group / 8 + n_items + 1
    unsigned char* rows;                         // [heads][tiles][TILE_BYTES]
    float2* factors;                             // [heads][tiles][8]: a row's factor, and its sum times that
    float2* norms;                               // [heads][tiles][8]: m, and 1 / sum (0 for a row that sees nothing)
    float2* parts;                               // [blocks][2][max_rows]: m and the sum, of segments that several blocks share
    KvJoin* joins;
    long long max_rows;
    float* scores;                               // [n_items][heads][width][score_rows]; null: they are found again in the second pass
    int score_rows;
    const float* base;
    float* mass;
    long long width;
    float decay;
};

// Where an item's tiles of 8 rows begin: items never overlap, whatever their sizes.
__device__ __forceinline__ long long tile_of(const MassArgs& P, int head, int item, int first)
{
    return head * P.tiles + (((long long)first * P.a.group) >> 3) + item;
}

// ---- query rows: a warp four heads of a token, eight lanes a row ----
// Integers of a tile: pieces (upper byte first), then [2][8 rows][4][16 bytes]: the bytes that a thread of the product needs are one load.
__global__ __launch_bounds__(256) void k_kv_mass_rows(const __grid_constant__ MassArgs P)
{
    kv_wait_before();
    kv_let_next();
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
    const long long tile = tile_of(P, kvh, item, x.first) + (r >> 3);
    unsigned char* to = P.rows + tile * TILE_BYTES + (r & 7) * 64;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        unsigned b[PIECES][2] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {            // even coordinates in the first word, odd ones in the second
            const int v = q[8 * half + i], low = (int)(signed char)v, v1 = (v - low) >> 8, mid = (int)(signed char)v1, high = (v1 - mid) >> 8;
            const int s = 8 * (i >> 1);
            b[0][i & 1] |= (unsigned)(high & 255) << s;
            b[1][i & 1] |= (unsigned)(mid & 255) << s;
            b[2][i & 1] |= (unsigned)(low & 255) << s;
        }
        const int c8 = 8 * half + l8;            // coordinates 8 c8 .. : word c8 & 3 of 16 bytes of codes, which lane c8 >> 2 has
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            *reinterpret_cast<uint2*>(to + p * 1024 + ((c8 >> 1) & 1) * 512 + (c8 >> 2) * 16 + (c8 & 1) * 8) = make_uint2(b[p][0], b[p][1]);
    }
    if (l8 == 0) {
        const float f = m * (A.scale * (KV_NORM * 1.4426950408889634f / TOP)) + wrong;
        P.factors[tile * 8 + (r & 7)] = make_float2(f, (float)sum * f);
    }
}

template <bool ASYM, int TILES>
struct alignas(16) Smem {
    static constexpr int PASS = TILES * TILE;
    unsigned char k[STAGES][UNIT * KV_ROW];
    float s[STAGES][UNIT * (ASYM ? 2 : 1)];
    unsigned there[STAGES][WARPS];               // which tokens have a page
    unsigned char q[TILES][TILE_BYTES];
    float2 factor[PASS];
    float2 norm[PASS];
    int lo[PASS], hi[PASS];
    float2 sum[WARPS][PASS];
    KvSeg seg;
    long long share[WARPS];
};

__device__ __forceinline__ void mma_s8(int c[4], const unsigned a[4], unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from)
{
    const unsigned dst = (unsigned)__cvta_generic_to_shared(to);
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ float2 norm_of(float m, float sum) { return sum == 0.f ? make_float2(0.f, 0.f) : make_float2(m, 1.f / sum); }
__device__ __forceinline__ float no_inf(float x) { return fmaf(x, 0.f, x); }

// MASS: the second pass.  KEEP: the first pass, which leaves the scores for k_kv_mass_sums.  TILES: taken at a time; one where no item has more than 8 rows of a KV head, which
// leaves registers enough (23.2 us instead of 25 with two).  Page numbers looked up a unit ahead: 24.1; four stages: 23.6.
template <bool ASYM, bool MASS, bool KEEP, int TILES>
__global__ __launch_bounds__(THREADS, BLOCKS_PER_SM) void k_kv_mass(const __grid_constant__ MassArgs P)
{
    constexpr int PART = MASS ? KV_ALL : KV_WHOLE, PASS = TILES * TILE;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<ASYM, TILES>& S = *reinterpret_cast<Smem<ASYM, TILES>*>(smem_raw);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, g = lane >> 2, t = lane & 3;
    kv_wait_before();
    kv_let_next();
    const int places = kv_share<THREADS, PART>(A, P.line, &S.seg, S.share);
    if (!MASS && tid == 0 && P.line.pad >= 0) P.joins[blockIdx.x] = KvJoin{0, 0, 0, 0};
    if (places == 0) return;

    KvSeg seg = S.seg;
    const int ps_log = A.c.page_log, ps = 1 << ps_log;
    for (bool more = true; more;) {
        const KvPiece piece = kv_piece(P.line, seg, places);
        const KvEntry& e = seg.e;
        const int n = max(piece.n, 0), tok_at = ((e.lo >> 7) + piece.skip) * UNIT;
        const int passes = TILES == 1 ? 1 : (e.rows + PASS - 1) / PASS;
        // what any row sees
        const int see_lo = kv_row_lo(A, e, 0), see_hi = kv_row_hi(A, e, A.by_group(e.rows - 1));
        const int* pages = A.c.page_table + (long long)e.seq * A.c.max_pages;
        const long long tile0 = tile_of(P, seg.head, seg.index, e.first);
        float* scores = KEEP ? P.scores + ((long long)seg.index * A.c.heads + seg.head) * P.width * P.score_rows : nullptr;

        // this thread's pieces of a unit: 16 bytes of the codes of tokens tid / 4 + 32 k, the scales of token tid
        const auto seen = [&](int tok) { return tok < see_hi && tok + UNIT > see_lo; };
        const auto fetch = [&](int i) {
            const int tok = tok_at + i * UNIT, st = i % STAGES;
            if (i < n && seen(tok)) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int pos = tok + (tid >> 2) + 32 * k, id = pos < see_hi ? pages[pos >> ps_log] : -1;
                    if ((unsigned)id < (unsigned)A.c.n_pages)
                        copy_async<16>(&S.k[st][((tid >> 2) + 32 * k) * KV_ROW + 16 * (tid & 3)],
                                       kv_block(A.c, id, seg.head) + (pos & (ps - 1)) * KV_ROW + 16 * (tid & 3));
                }
                const int pos = tok + tid, id = pos < see_hi ? pages[pos >> ps_log] : -1;
                const bool ok = (unsigned)id < (unsigned)A.c.n_pages;
                if (ok) copy_async<ASYM ? 8 : 4>(&S.s[st][tid * (ASYM ? 2 : 1)], kv_block(A.c, id, seg.head) + 2 * ps * KV_ROW + (pos & (ps - 1)) * (ASYM ? 8 : 4));
                const unsigned there = __ballot_sync(0xffffffffu, ok);
                if (lane == 0) S.there[st][w] = there;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // the rows of a pass, into registers and then into shared memory
        constexpr int PER = TILE_BYTES / 16, LOADS = (TILES * PER + THREADS - 1) / THREADS;
        uint4 qv[LOADS];
        float2 fv = make_float2(0.f, 0.f);
        float2 nv = make_float2(0.f, 0.f);
        int lov = 0, hiv = 0;
        const auto load_rows = [&](int pass) {
            const uint4* from = reinterpret_cast<const uint4*>(P.rows + (tile0 + TILES * pass) * TILE_BYTES);
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int i = tid + THREADS * k;
                if (i < TILES * PER && TILE * (i / PER) + PASS * pass < e.rows) qv[k] = __ldg(from + i);
            }
            const int r = PASS * pass + tid;
            fv = make_float2(0.f, 0.f);
            nv = make_float2(0.f, 0.f);
            lov = hiv = 0;
            if (tid < PASS && r < e.rows) {
                fv = P.factors[tile0 * 8 + r];
                if (MASS) nv = P.norms[tile0 * 8 + r];
                const int token = A.by_group(r);
                lov = kv_row_lo(A, e, token);
                hiv = kv_row_hi(A, e, token);
            }
        };
        const auto store_rows = [&] {
#pragma unroll
            for (int k = 0; k < LOADS; ++k)
                if (tid + THREADS * k < TILES * PER) reinterpret_cast<uint4*>(S.q[0])[tid + THREADS * k] = qv[k];
            if (tid < PASS) {
                S.factor[tid] = fv;
                S.norm[tid] = nv;
                S.lo[tid] = lov;
                S.hi[tid] = hiv;
            }
        };

        load_rows(0);
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) fetch(i);
        __syncthreads();                         // the segment before is done with the rows
        store_rows();
        float m[TILES][2], l[TILES][2];
        const auto reset = [&] {
#pragma unroll
            for (int i = 0; i < TILES; ++i) m[i][0] = m[i][1] = NONE, l[i][0] = l[i][1] = 0.f;
        };
        reset();
        // (m, sum) of the block's rows of a pass, with what was there before in `slot`
        float2* slot = P.parts + ((long long)blockIdx.x * 2 + (piece.starts ? 1 : 0)) * P.max_rows;
        const auto reduce = [&](int pass, bool first, bool last) {
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float top = m[i][j];
#pragma unroll
                    for (int h = 4; h < 32; h <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, h));
                    float s = l[i][j] * kv_ex2(m[i][j] - top);
#pragma unroll
                    for (int h = 4; h < 32; h <<= 1) s += __shfl_xor_sync(0xffffffffu, s, h);
                    if (g == 0) S.sum[w][TILE * i + 2 * t + j] = make_float2(top, s);
                }
            __syncthreads();
            const int r = PASS * pass + tid;
            if (tid < PASS && r < e.rows) {
                float2 x = first ? make_float2(NONE, 0.f) : slot[r];
#pragma unroll
                for (int i = 0; i < WARPS; ++i) {
                    const float2 y = S.sum[i][tid];
                    const float top = fmaxf(x.x, y.x);
                    x.y = x.y * kv_ex2(x.x - top) + y.y * kv_ex2(y.x - top);
                    x.x = top;
                }
                if (last && piece.starts && piece.ends) P.norms[tile0 * 8 + r] = norm_of(x.x, x.y);
                else slot[r] = x;
            }
        };

        for (int u = 0; u < n; ++u) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncthreads();
            fetch(u + STAGES - 1);
            const int st = u % STAGES, tok0 = tok_at + u * UNIT, mine = tok0 + 32 * w;
            float acc[2][2] = {}, off[2][2] = {};        // sums over thousands of rows, with what their rounding has left out
            if (seen(tok0)) {
                // this thread's codes: of tokens 16 h + g and 8 further, and their scales
                unsigned a[2][4][4];
                float ks[2][2], km[2][2];
                const unsigned there = S.there[st][w];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int at = 32 * w + 16 * h + 8 * b + g;
                        const uint4 c = *reinterpret_cast<const uint4*>(&S.k[st][at * KV_ROW + 16 * t]);
                        const unsigned v[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const unsigned x = ASYM ? v[i] ^ 0x88888888u : v[i];
                            a[h][i][b] = (x << 4) & 0xf0f0f0f0u;
                            a[h][i][2 + b] = x & 0xf0f0f0f0u;
                        }
                        if (ASYM) {
                            const float2 x = *reinterpret_cast<const float2*>(&S.s[st][2 * at]);
                            ks[h][b] = no_inf(fmaf(x.y, 0.f, x.x)) * 0.0625f;
                            km[h][b] = fmaf(8.f, x.x, x.y);
                        } else {
                            ks[h][b] = no_inf(S.s[st][at]) * 0.0625f;
                            km[h][b] = 0.f;
                        }
                    }
                for (int pass = 0; pass < passes; ++pass) {
                    if (passes > 1) load_rows(pass + 1 < passes ? pass + 1 : 0);
                    const int last = min(e.rows, PASS * (pass + 1)) - 1;
                    const int pass_lo = kv_row_lo(A, e, A.by_group(PASS * pass)), pass_hi = kv_row_hi(A, e, A.by_group(last));
                    if (mine < pass_hi && mine + 32 > pass_lo) {
                        const bool plain = there == 0xffffffffu && mine >= kv_row_lo(A, e, A.by_group(last)) && mine + 32 <= kv_row_hi(A, e, A.by_group(PASS * pass));
                        float got[2][2] = {};
#pragma unroll
                        for (int i = 0; i < TILES; ++i) {
                            if (i > 0 && PASS * pass + TILE * i >= e.rows) break;
                            int c[2][PIECES][4] = {};
#pragma unroll
                            for (int p = 0; p < PIECES; ++p)
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const uint4 b = *reinterpret_cast<const uint4*>(&S.q[i][p * 1024 + k * 512 + g * 64 + t * 16]);
#pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        mma_s8(c[h][p], a[h][2 * k], b.x, b.y);
                                        mma_s8(c[h][p], a[h][2 * k + 1], b.z, b.w);
                                    }
                                }
                            const float4 f = *reinterpret_cast<const float4*>(&S.factor[TILE * i + 2 * t]);         // rows 2 t and 2 t + 1
                            const float4 norm = MASS ? *reinterpret_cast<const float4*>(&S.norm[TILE * i + 2 * t]) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const int2 lo = *reinterpret_cast<const int2*>(&S.lo[TILE * i + 2 * t]), hi = *reinterpret_cast<const int2*>(&S.hi[TILE * i + 2 * t]);
                            float z[2][4];
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float x = fmaf((float)(256 * c[h][0][j] + c[h][1][j]), 256.f, (float)c[h][2][j]);
                                    const float fac = j & 1 ? f.z : f.x, lift = j & 1 ? f.w : f.y;
                                    z[h][j] = fmaf(x, ks[h][j >> 1] * fac, ASYM ? km[h][j >> 1] * lift : 0.f);
                                    if (MASS) z[h][j] = __fsub_rn(z[h][j], j & 1 ? norm.z : norm.x);         // from the score as the first pass had it, to the last bit
                                    if (!plain) {
                                        const int pos = mine + 16 * h + 8 * (j >> 1) + g;
                                        if (pos < (j & 1 ? lo.y : lo.x) || pos >= (j & 1 ? hi.y : hi.x) || !(there >> (16 * h + 8 * (j >> 1) + g) & 1)) z[h][j] = -INFINITY;
                                    }
                                }
                            const int row = PASS * pass + TILE * i + 2 * t;
                            if (KEEP && row < P.score_rows)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
#pragma unroll
                                    for (int b = 0; b < 2; ++b) {
                                        const int pos = mine + 16 * h + 8 * b + g;
                                        if (pos < P.width) *reinterpret_cast<float2*>(scores + (long long)pos * P.score_rows + row) = make_float2(z[h][2 * b], z[h][2 * b + 1]);
                                    }
                            if (MASS) {
#pragma unroll
                                for (int h = 0; h < 2; ++h)
#pragma unroll
                                    for (int j = 0; j < 4; ++j) got[h][j >> 1] = fmaf(kv_ex2(z[h][j]), j & 1 ? norm.w : norm.y, got[h][j >> 1]);
                            } else {
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const float top = fmaxf(fmaxf(z[0][j], z[0][j + 2]), fmaxf(z[1][j], z[1][j + 2]));
                                    if (top > m[i][j] + MOVE) {
                                        const float whole = ceilf(top);          // so that sums change by exact powers of two
                                        l[i][j] *= kv_ex2(m[i][j] - whole);
                                        m[i][j] = whole;
                                    }
                                    l[i][j] += (kv_ex2(z[0][j] - m[i][j]) + kv_ex2(z[0][j + 2] - m[i][j])) + (kv_ex2(z[1][j] - m[i][j]) + kv_ex2(z[1][j + 2] - m[i][j]));
                                }
                            }
                        }
                        if (MASS) {
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const float y = __fsub_rn(got[h][b], off[h][b]), sum = __fadd_rn(acc[h][b], y);
                                    off[h][b] = __fsub_rn(__fsub_rn(sum, acc[h][b]), y);
                                    acc[h][b] = sum;
                                }
                        }
                    }
                    if (passes > 1) {
                        if (!MASS) {
                            reduce(pass, u == 0, u + 1 == n);
                            reset();
                        }
                        __syncthreads();
                        store_rows();
                        __syncthreads();
                    }
                }
            } else if (!MASS && passes > 1 && u == 0) {          // the only unit of rows that see nothing
                for (int pass = 0; pass < passes; ++pass) {
                    reduce(pass, true, n == 1);
                    __syncthreads();
                }
            }
            if (MASS) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        acc[h][b] += __shfl_xor_sync(0xffffffffu, acc[h][b], 1);
                        acc[h][b] += __shfl_xor_sync(0xffffffffu, acc[h][b], 2);
                        const int pos = mine + 16 * h + 8 * b + g;
                        if (t == 0 && pos < e.length && pos < P.width) {
                            const long long at = ((long long)e.seq * A.c.heads + seg.head) * P.width + pos;
                            P.mass[at] = pos < e.before && P.decay != 0.f ? fmaf(P.decay, P.base[at], acc[h][b]) : acc[h][b];
                        }
                    }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (!MASS) {
            if (passes == 1 && n > 0) reduce(0, true, true);
            if (tid == 0 && n > 0 && piece.starts && !piece.ends) P.joins[blockIdx.x] = kv_join(P.line, seg, places);
        }
        more = kv_more(P.line, seg, places);
        __syncthreads();                         // the stages and the sums may be written again
        if (more) kv_next<PART>(A, P.line, seg);
    }
}

// The sums of rows whose segments several blocks share: block b joins the one that starts in block b of the pass before.
__global__ __launch_bounds__(128) void k_kv_mass_join(const __grid_constant__ MassArgs P)
{
    kv_wait_before();
    kv_let_next();
    const KvJoin j = P.joins[blockIdx.x];
    if (j.blocks == 0) return;
    const KvEntry e = kv_entry(P.a, P.line, j.index);
    const long long tile0 = tile_of(P, j.head, j.index, e.first);
    const float2* first = P.parts + ((long long)blockIdx.x * 2 + 1) * P.max_rows;
    for (int r = threadIdx.x + 128 * blockIdx.y; r < e.rows; r += 128 * gridDim.y) {
        float top = NONE, sum = 0.f;
        for (int b = 0; b < j.blocks; ++b) {
            const float2 x = (b == 0 ? first : first + (long long)(2 * b - 1) * P.max_rows)[r];
            const float now = fmaxf(top, x.x);
            sum = sum * kv_ex2(top - now) + x.y * kv_ex2(x.x - now);
            top = now;
        }
        P.norms[tile0 * 8 + r] = norm_of(top, sum);
    }
}

// The second pass from scores that the first one left: a thread a position, four of a thread's on their way at once (one: 14 us instead of 8 for 830 000 tokens and KV heads).
constexpr int SUMS = 4 * 256;
__global__ __launch_bounds__(256) void k_kv_mass_sums(const __grid_constant__ MassArgs P)
{
    __shared__ float2 norm[GBS_KV_MASS_FEW_ROWS];
    __shared__ int2 sees[GBS_KV_MASS_FEW_ROWS];
    kv_wait_before();
    kv_let_next();
    const gbs_kv_attn& A = P.a;
    const int item = blockIdx.x / A.c.heads, head = blockIdx.x - item * A.c.heads;
    const KvEntry e = kv_entry<KV_ALL>(A, P.line, item);
    if (e.units == 0 || (long long)SUMS * blockIdx.y >= e.length) return;
    if (threadIdx.x < e.rows) {
        const int token = A.by_group(threadIdx.x);
        norm[threadIdx.x] = P.norms[tile_of(P, head, item, e.first) * 8 + threadIdx.x];
        sees[threadIdx.x] = make_int2(kv_row_lo(A, e, token), kv_row_hi(A, e, token));
    }
    __syncthreads();
    const long long row = ((long long)e.seq * A.c.heads + head) * P.width;
    const int most = (int)min((long long)e.length, P.width);
    for (long long first = (long long)SUMS * blockIdx.y; first < most; first += (long long)SUMS * gridDim.y) {
        float sum[4], old[4];
        int pos[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            pos[k] = (int)first + 256 * k + (int)threadIdx.x;
            sum[k] = 0.f;
            old[k] = P.decay != 0.f && pos[k] < min(most, e.before) ? P.base[row + pos[k]] : 0.f;
        }
        const float* z = P.scores + ((long long)item * A.c.heads + head) * P.width * P.score_rows;
        const auto add = [&](int k, int r, float x) {
            const float2 n = norm[r];
            const int2 s = sees[r];
            if (r < e.rows && pos[k] >= s.x && pos[k] < s.y) sum[k] = fmaf(kv_ex2(x - n.x), n.y, sum[k]);
        };
        if ((P.score_rows & 3) == 0) {
            for (int r = 0; r < e.rows; r += 4) {
                float4 x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (pos[k] < most) x[k] = *reinterpret_cast<const float4*>(z + (long long)pos[k] * P.score_rows + r);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    add(k, r, x[k].x);
                    add(k, r + 1, x[k].y);
                    add(k, r + 2, x[k].z);
                    add(k, r + 3, x[k].w);
                }
            }
        } else {
            for (int r = 0; r < e.rows; r += 2) {
                float2 x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (pos[k] < most) x[k] = *reinterpret_cast<const float2*>(z + (long long)pos[k] * P.score_rows + r);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    add(k, r, x[k].x);
                    add(k, r + 1, x[k].y);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (pos[k] < most) P.mass[row + pos[k]] = fmaf(P.decay, old[k], sum[k]);
    }
}

int tiles_of(const gbs_kv_attn& A) { return std::min<int64_t>(A.max_tokens, A.n_tokens) * A.group <= TILE ? 1 : 2; }
int blocks_of(const gbs_plan* p) { return p->sm_count * BLOCKS_PER_SM; }
int64_t round_up(int64_t x) { return (x + 15) & ~(int64_t)15; }

struct Layout {
    int64_t tiles, max_rows, rows, factors, norms, parts, joins, scores, bytes;
    int score_rows;                              // 0: scores are not kept
};
// Keeping scores (4 bytes a row, token and KV head, written once and read once) takes less time than finding them again from the keys, but room by the width, since the
// lengths are not known here: up to this many bytes.
constexpr int64_t MOST_SCORES = 256ll << 20;

Layout layout_of(const gbs_plan* p, const gbs_kv_attn& A, int64_t width)
{
    Layout l;
    l.tiles = A.n_tokens * A.group / 8 + A.n_items + 1;
    l.max_rows = (int64_t)std::min<int64_t>(A.max_tokens, A.n_tokens) * A.group;
    l.rows = 0;
    l.factors = round_up(A.c.heads * l.tiles * TILE_BYTES);
    l.norms = l.factors + round_up(A.c.heads * l.tiles * 8 * (int64_t)sizeof(float2));
    l.parts = l.norms + round_up(A.c.heads * l.tiles * 8 * (int64_t)sizeof(float2));
    l.joins = l.parts + round_up((int64_t)blocks_of(p) * 2 * l.max_rows * sizeof(float2));
    l.scores = l.joins + round_up((int64_t)blocks_of(p) * sizeof(KvJoin));
    const int64_t rows = (l.max_rows + 1) & ~1ll, places = (int64_t)A.n_items * A.c.heads * rows * (int64_t)sizeof(float);
    l.score_rows = places > 0 && width <= MOST_SCORES / places ? (int)rows : 0;
    l.bytes = l.scores + (l.score_rows ? places * width : 0);
    return l;
}

template <bool MASS, bool KEEP, int TILES>
int launch(const gbs_plan* p, const MassArgs& P, cudaStream_t stream)
{
    const auto f = p->asym ? k_kv_mass<true, MASS, KEEP, TILES> : k_kv_mass<false, MASS, KEEP, TILES>;
    const size_t smem = p->asym ? sizeof(Smem<true, TILES>) : sizeof(Smem<false, TILES>);
    const cudaError_t e = cudaFuncSetAttribute((const void*)f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return e != cudaSuccess ? (int)e : gbs_kv_launch(p, f, dim3((unsigned)blocks_of(p)), THREADS, smem, stream, P);
}
template <bool MASS, bool KEEP>
int launch(const gbs_plan* p, const MassArgs& P, cudaStream_t stream)
{
    return tiles_of(P.a) == 1 ? launch<MASS, KEEP, 1>(p, P, stream) : launch<MASS, KEEP, 2>(p, P, stream);
}

bool many(const gbs_kv_attn& A) { return std::min<int64_t>(A.max_tokens, A.n_tokens) * A.group > GBS_KV_MASS_FEW_ROWS; }

}  // namespace

int64_t gbs_kv_mass_workspace(const gbs_plan* p, const gbs_kv_attn& A, int64_t width) { return many(A) ? gbs_tc_kvmass_workspace(p, A, width) : layout_of(p, A, width).bytes; }

int gbs_kv_mass_launch(const gbs_plan* p, const gbs_kv_attn& A, const float* base, float decay, float* mass, int64_t width, void* workspace,
                       cudaStream_t stream)
{
    if (many(A)) return gbs_tc_kvmass_launch(p, A, base, decay, mass, width, workspace, stream);
    const Layout l = layout_of(p, A, width);
    unsigned char* w = static_cast<unsigned char*>(workspace);
    MassArgs P = {};
    P.a = A;
    P.line.tile_rows = 1 << 29;                  // an item is one tile
    P.line.unit_log = 7;
    P.line.tiles = 1;
    P.line.by_tiles.set(1);
    P.line.entries = A.n_items;
    P.line.pad = 2;
    P.line.least = 2;
    P.tiles = l.tiles;
    P.rows = w + l.rows;
    P.factors = reinterpret_cast<float2*>(w + l.factors);
    P.norms = reinterpret_cast<float2*>(w + l.norms);
    P.parts = reinterpret_cast<float2*>(w + l.parts);
    P.joins = reinterpret_cast<KvJoin*>(w + l.joins);
    P.max_rows = l.max_rows;
    P.scores = reinterpret_cast<float*>(w + l.scores);
    P.score_rows = l.score_rows;
    P.base = base;
    P.mass = mass;
    P.width = width;
    P.decay = decay;
    const int64_t jobs = A.n_tokens * ((A.n_heads + 3) / 4);
    int rc = gbs_kv_launch(p, k_kv_mass_rows, dim3((unsigned)((jobs + 7) / 8)), 256, 0, stream, P);
    const bool keep = l.score_rows > 0;
    if (rc == 0) rc = keep ? launch<false, true>(p, P, stream) : launch<false, false>(p, P, stream);
    const unsigned y = (unsigned)std::min<int64_t>((l.max_rows + 127) / 128, 64);
    if (rc == 0) rc = gbs_kv_launch(p, k_kv_mass_join, dim3((unsigned)blocks_of(p), y), 128, 0, stream, P);
    if (rc != 0) return rc;
    if (!keep) return launch<true, false>(p, P, stream);
    return gbs_kv_launch(p, k_kv_mass_sums, dim3((unsigned)A.n_items * (unsigned)A.c.heads, (unsigned)std::min<int64_t>((width + SUMS - 1) / SUMS, 4096)), 256, 0, stream, P);
}
