// Attention over the paged KV cache for prompts and chunks of them (gbs_kv_attention, more than 16 query rows of an item and KV head), on
// tcgen05: tiles of 128 rows (tokens x query heads of a KV head) by 128 cached tokens.
//
// The mathematics is that of gbs_kv_attn.cu: codes enter the matrix unit as they are (exact in fp16), scales stay outside.
//     S = Q C_k^T (fp16, fp32 sums),  z = S Delta_k f + log2 Delta_v,  w = 2^(z - M + 6),  O += w C_v,  l += w / Delta_v.
// With log2 Delta_v inside the exponent one running maximum M (of z) serves both the weights' range in fp16 and the softmax; a row with zero
// values alone has codes 0, and takes the largest scale next to it.  f is the row's factor (its power of two, the softmax scale).
//
// All eight warps do the same in turn: the softmax of 16 rows (a thread has two of them and every fourth pair of columns, so that a tile's per-token
// numbers are read once for 16 rows), then half a row of key codes and half a row of value codes of the next tile to fp16, fetched
// into registers a tile ahead.  Warp 0 also issues the MMAs.  Scores and weights share 128 columns of tensor memory (a warp's
// fp16 weights overwrite scores it has read), the sums take 128 more, so two blocks run on an SM and fill each other's gaps.
// A tile's work on an SM: 2 x 512 cycles of MMA, 1024 of ex2, about 1700 of instructions issued.  It takes 3200: no unit is more than half
// busy, and what bounds it is the chain of latencies of a tile (scores, softmax, weights, second product) with only two blocks to overlap.  The
// last 2048 of 8048 tokens, 32 query heads over 8 KV heads, take 433 us, 545 TFLOP/s.  Four more warps for the codes (80 registers a thread) took
// 447 us, tiles of 64 tokens with two sets of scores 567 us, scalar arithmetic instead of pairs the same time.
// fp16 weights reach 2^-30 of the largest w, below what a bf16 result shows.  l is of fp32 weights over Delta_v, which go under when value
// scales that one row sees differ by more than 2^100: the share of the small ones in l is then lost.
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
    int lo[ROWS], hi[ROWS];                          // tokens that a row sees
    float m[ROWS], l[ROWS], add[ROWS];
    unsigned long long block[3][UNIT / 16];          // of tile i in [i % 3]: where the blocks of its pages are; bit 0: there is none
    unsigned long long kfull, vfull, vfree, sfull, pfull;
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
// 16 lanes: thread T has rows T / 4 and T / 4 + 8; of each 8 columns 2 (T % 4) and the next one (registers 4 i, 4 i + 1 of the upper row,
// 4 i + 2, 4 i + 3 of the lower), of each 4 columns T % 4 (registers 2 i and 2 i + 1)
__device__ __forceinline__ void tmem_ld64(unsigned taddr, unsigned r[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st64(unsigned taddr, const unsigned r[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x8.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld32p(unsigned taddr, unsigned r[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x128b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32p(unsigned taddr, const unsigned r[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// byte of a 16-byte piece (8 coordinates) of a row in a tile
__device__ __forceinline__ unsigned piece_at(int row, int piece)
{
    return (unsigned)(piece >> 3) * (128 * 128) + (unsigned)(row >> 3) * 1024 + (unsigned)(row & 7) * 128 + (unsigned)(((piece & 7) ^ (row & 7)) << 4);
}
// byte of a 16-byte piece (4 coordinates) of a row of sums
__device__ __forceinline__ unsigned sum_at(int row, int piece) { return (unsigned)row * 512 + (unsigned)((piece ^ (row & 31)) << 4); }

// Half of a cached token's codes (64 coordinates) and its scales on their way through registers.
struct Token {
    uint4 k[2], v[2];
    float ks, kl, vs, vl;
    bool ok;
};

// Where the block of a page is, bit 0 set for a page that is none: some block of the pool then, whose codes will weigh nothing.
__device__ __forceinline__ unsigned long long block_of(const gbs_kv_attn& A, const KvSeg& s, int page)
{
    const bool ok = (unsigned)page < (unsigned)A.c.n_pages;
    return reinterpret_cast<unsigned long long>(kv_block(A.c, ok ? page : 0, s.head)) | (ok ? 0ull : 1ull);
}
// `at`: this thread's codes in a block
template <bool ASYM>
__device__ __forceinline__ void load_k(Token& x, const unsigned char* block, int at, int slot, int ps)
{
    const uint4* c = reinterpret_cast<const uint4*>(block + at);
    x.k[0] = c[0];
    x.k[1] = c[1];
    x.kl = x.vl = 0.f;
    const float* sc = reinterpret_cast<const float*>(block + 2 * ps * KV_ROW);
    if (ASYM) {
        const float2 a = reinterpret_cast<const float2*>(sc)[slot], b = reinterpret_cast<const float2*>(sc)[ps + slot];
        x.ks = a.x; x.kl = a.y; x.vs = b.x; x.vl = b.y;
    } else {
        x.ks = sc[slot];
        x.vs = sc[ps + slot];
    }
}
__device__ __forceinline__ void load_v(Token& x, const unsigned char* block, int at)
{
    const uint4* c = reinterpret_cast<const uint4*>(block + at);
    x.v[0] = c[0];
    x.v[1] = c[1];
}
template <bool ASYM>
__device__ __forceinline__ void store_codes(unsigned char* tile, int row, int half, const uint4 c[2])
{
    const unsigned first = smem_u32(tile) + piece_at(row, 8 * half);     // a tile starts on 1024 bytes: the piece's number is exclusive-or'ed in
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 q = c[i >> 2];
        const unsigned w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
        unsigned h[4];
        kv_codes_f16<ASYM>(w, h);
        st_shared_v4(first ^ (unsigned)(i << 4), make_uint4(h[0], h[1], h[2], h[3]));
    }
}

// What a warp's 16 rows have added up, and the weights of the first half of the tile, times a factor of each row; rare.
__device__ __forceinline__ void shrink(unsigned lanes, float keep_a, float keep_b, bool sums, bool weights)
{
    tmem_st_wait();
    if (sums) {
#pragma unroll 1
        for (int q = 0; q < 2; ++q) {
            unsigned o[32];
            tmem_ld64(lanes + O_COL + 64 * q, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * ((k & 2) ? keep_b : keep_a));
            tmem_st64(lanes + O_COL + 64 * q, o);
        }
    }
    if (weights) {
        unsigned o[16];
        tmem_ld32p(lanes, o);
        const __half2 ha = __float2half2_rn(keep_a), hb = __float2half2_rn(keep_b);
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = as_u(__hmul2(as_h(o[k]), (k & 1) ? hb : ha));
        tmem_st32p(lanes, o);
    }
}

template <bool ASYM>
__global__ __launch_bounds__(THREADS, BLOCKS_PER_SM) void k_tc_kvattn(const __grid_constant__ KvAttnArgs P)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const gbs_kv_attn& A = P.a;
    const int tid = threadIdx.x, lane = tid & 31, w = warp_index();
    if (tid == 0) {
        S.abort = 0;
        mbar_init(&S.kfull, 8);
        mbar_init(&S.vfull, 8);
        mbar_init(&S.vfree, 1);
        mbar_init(&S.sfull, 1);
        mbar_init(&S.pfull, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == 0) tmem_alloc(&S.tmem, TMEM_COLS);
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
        const int me = tid & 127, part = tid >> 7;           // this thread's token of a tile, and which half of its row
        const int slot = me & (ps - 1), my_page = me >> ps_log, k_at = slot * KV_ROW + 32 * part, v_at = k_at + ps * KV_ROW;     // the same in every tile
        const int* row_of_pages = A.c.page_table + (long long)seg.e.seq * A.c.max_pages;
        const auto page_of = [&](int tok) { return tok < seg.e.hi ? row_of_pages[tok >> ps_log] : -1; };
        const auto seen = [&](unsigned long long b, int tok) { return !(b & 1) && tok >= seg.e.lo && tok < seg.e.hi; };
        unsigned long long here = block_of(A, seg, page_of(tok0 + me));
        const unsigned char* block = reinterpret_cast<const unsigned char*>(here & ~1ull);
        x.ok = seen(here, tok0 + me);
        load_k<ASYM>(x, block, k_at, slot, ps);
        load_v(x, block, v_at);
        // warp 7, a lane a page: the blocks of the tiles ahead
        int page = -1;
        if (w == 7 && lane < (UNIT >> ps_log)) {
            S.block[1][lane] = block_of(A, seg, page_of(tok0 + UNIT + (lane << ps_log)));
            page = page_of(tok0 + 2 * UNIT + (lane << ps_log));
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
                    const int token = A.by_group(min(seg.e.row0 + row, seg.e.rows - 1));
                    S.lo[row] = kv_row_lo(A, seg.e, token);
                    S.hi[row] = seg.e.row0 + row < seg.e.rows ? kv_row_hi(A, seg.e, token) : 0;
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();

        constexpr unsigned ID_S = (1u << 4) | ((unsigned)(UNIT >> 3) << 17) | ((unsigned)(ROWS >> 4) << 24);             // fp16, both K-major
        constexpr unsigned ID_O = ID_S | (1u << 16);                                                                    // B N-major
        // the keys of tile i into shared memory, those of tile i + 1 on their way.  The tile before has been read: its scores are there
        const auto keys = [&](int i) {
            const int tok = tok0 + i * UNIT + me, b = (it + i) & 1;
            // zero rows take the largest scale next to them; tokens that are not there weigh nothing, and scales that are no
            // numbers make the scores of those that see them none
            if (part == 0) {
                float vs = x.ok ? x.vs : 0.f;
                const float near = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(vs) & 0x7fffffffu));
                const bool wrong = x.ok && (!(fabsf(vs) < INFINITY) || !(fabsf(x.vl) < INFINITY));
                if (vs == 0.f) vs = near > 0.f && near < INFINITY ? near : 1.f;
                vs = fmaxf(vs, 7.888609052210118e-31f);                          // 2^-100
                S.lv[b][me] = !x.ok ? -INFINITY : wrong ? NAN : __log2f(vs);
                S.rv[b][me] = x.ok && !wrong ? __fdividef(1.f, vs) : 0.f;
                if (ASYM) S.vl[b][me] = wrong || !x.ok ? 0.f : x.vl;
            } else {
                S.ks[b][me] = x.ok ? x.ks : 0.f;
                if (ASYM) S.kl[b][me] = x.ok ? x.kl : 0.f;
                if (w == 7 && lane < (UNIT >> ps_log)) {
                    S.block[(unsigned)(i + 2) % 3u][lane] = block_of(A, seg, page);
                    page = page_of(tok0 + (i + 3) * UNIT + (lane << ps_log));
                }
            }
            store_codes<ASYM>(S.k, me, part, x.k);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.kfull);
            const unsigned long long e = S.block[(unsigned)(i + 1) % 3u][my_page];
            block = reinterpret_cast<const unsigned char*>(e & ~1ull);
            x.ok = seen(e, tok + UNIT);
            load_k<ASYM>(x, block, k_at, slot, ps);
        };
        const auto values = [&](int i, const unsigned char* next_block) {
            store_codes<ASYM>(S.v, me, part, x.v);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.vfull);
            load_v(x, next_block, v_at);
        };
        const auto scores = [&](int i) {
            if (!mbar_wait_warp(&S.abort, &S.kfull, (it + i) & 1u, P.status, 71)) return false;
            tc_fence_after();
            const unsigned long long qd = smem_desc(smem_u32(S.q), 16, 1024, 2), kd = smem_desc(smem_u32(S.k), 16, 1024, 2);
#pragma unroll
            for (int k = 0; k < 8; ++k) {                    // sixteen coordinates: 32 bytes, four of them in a block of 64
                const unsigned long long off = (unsigned)((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
                umma_f16(tmem, qd + off, kd + off, ID_S, k > 0);
            }
            umma_commit(&S.sfull);
            return true;
        };

        // this thread's rows: r0 and r0 + 8
        const int r0 = 32 * (w & 3) + 16 * (w >> 2) + (lane >> 2), c0 = 2 * (lane & 3);
        const unsigned lanes = tmem + ((unsigned)(32 * (w & 3) + 16 * (w >> 2)) << 16);
        const f32x2 fa = both(S.factor[r0]), fb = both(S.factor[r0 + 8]);
        const f32x2 qa = both(S.qsum[r0]), qb = both(S.qsum[r0 + 8]);
        // tokens that every row of the tile sees need no mask
        const int all_lo = kv_row_lo(A, seg.e, A.by_group(min(seg.e.rows, seg.e.row0 + ROWS) - 1)), all_hi = kv_row_hi(A, seg.e, A.by_group(seg.e.row0));
        float Ma = NONE, Mb = NONE;
        f32x2 la = both(0.f), lb = la, ea = la, eb = la;     // totals and sums of p lo, of even and odd columns
        keys(0);
        {
            const unsigned char* ahead = block;
            values(0, ahead);
        }
        bool ok = w != 0 || scores(0);
        for (int i = 0; i < n && ok; ++i) {
            const unsigned now = it + i;
            const int b = now & 1, tok = tok0 + i * UNIT;
            const bool plain = tok >= all_lo && tok + UNIT <= all_hi;
            if (!(ok = mbar_wait_warp(&S.abort, &S.sfull, now & 1u, P.status, 76))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {                    // 64 columns at a time
                unsigned r[32];
                tmem_ld64(lanes + 64 * c, r);
                tmem_ld_wait(r);
                const int at = 64 * c + c0;
                f32x2 z[16];                                 // of columns 8 j + c0, the next one: upper row, lower row
                float ta = NONE, tb = NONE;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const f32x2 k2 = *reinterpret_cast<const f32x2*>(&S.ks[b][at + 8 * j]), v2 = *reinterpret_cast<const f32x2*>(&S.lv[b][at + 8 * j]);
                    f32x2 u = mul2(pk(r[4 * j], r[4 * j + 1]), k2), d = mul2(pk(r[4 * j + 2], r[4 * j + 3]), k2);
                    if (ASYM) {
                        const f32x2 o2 = *reinterpret_cast<const f32x2*>(&S.kl[b][at + 8 * j]);
                        u = fma2(o2, qa, u);
                        d = fma2(o2, qb, d);
                    }
                    z[2 * j] = fma2(u, fa, v2);
                    z[2 * j + 1] = fma2(d, fb, v2);
                }
                if (!plain) {
                    const int loa = S.lo[r0], hia = S.hi[r0], lob = S.lo[r0 + 8], hib = S.hi[r0 + 8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        unsigned u0, u1;
                        const int t = tok + at + 8 * j;
                        unpk(z[2 * j], u0, u1);
                        if (t < loa || t >= hia) u0 = 0xff800000u;
                        if (t + 1 < loa || t + 1 >= hia) u1 = 0xff800000u;
                        z[2 * j] = pk(u0, u1);
                        unpk(z[2 * j + 1], u0, u1);
                        if (t < lob || t >= hib) u0 = 0xff800000u;
                        if (t + 1 < lob || t + 1 >= hib) u1 = 0xff800000u;
                        z[2 * j + 1] = pk(u0, u1);
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    unsigned u0, u1;
                    unpk(z[2 * j], u0, u1);
                    ta = max3(__uint_as_float(u0), __uint_as_float(u1), ta);
                    unpk(z[2 * j + 1], u0, u1);
                    tb = max3(__uint_as_float(u0), __uint_as_float(u1), tb);
                }
                if (__any_sync(0xffffffffu, ta > Ma + MOVE || tb > Mb + MOVE)) {
                    // rare: a row's four threads agree on its maximum, and what has been added up by the old one shrinks
#pragma unroll
                    for (int h = 1; h < 4; h <<= 1) {
                        ta = fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, h));
                        tb = fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, h));
                    }
                    ta = fmaxf(ta, Ma);
                    tb = fmaxf(tb, Mb);
                    const float keep_a = kv_ex2(Ma - ta), keep_b = kv_ex2(Mb - tb);
                    Ma = ta;
                    Mb = tb;
                    la = mul2(la, both(keep_a));
                    lb = mul2(lb, both(keep_b));
                    ea = mul2(ea, both(keep_a));
                    eb = mul2(eb, both(keep_b));
                    shrink(lanes, keep_a, keep_b, i > 0, c > 0);
                }
                const f32x2 base_a = both(6.f - Ma), base_b = both(6.f - Mb);        // weights are 64 at M
                unsigned st[16];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const f32x2 r2 = *reinterpret_cast<const f32x2*>(&S.rv[b][at + 8 * j]);
                    unsigned u0, u1, d0, d1;
                    unpk(add2(z[2 * j], base_a), u0, u1);
                    unpk(add2(z[2 * j + 1], base_b), d0, d1);
                    const float wa0 = kv_ex2(__uint_as_float(u0)), wa1 = kv_ex2(__uint_as_float(u1));
                    const float wb0 = kv_ex2(__uint_as_float(d0)), wb1 = kv_ex2(__uint_as_float(d1));
                    const f32x2 wa = pk(__float_as_uint(wa0), __float_as_uint(wa1)), wb = pk(__float_as_uint(wb0), __float_as_uint(wb1));
                    if (ASYM) {
                        const f32x2 o2 = *reinterpret_cast<const f32x2*>(&S.vl[b][at + 8 * j]);
                        const f32x2 pa = mul2(wa, r2), pb = mul2(wb, r2);
                        la = add2(la, pa);
                        lb = add2(lb, pb);
                        ea = fma2(pa, o2, ea);
                        eb = fma2(pb, o2, eb);
                    } else {
                        la = fma2(wa, r2, la);
                        lb = fma2(wb, r2, lb);
                    }
                    st[2 * j] = as_u(__floats2half2_rn(wa0, wa1));
                    st[2 * j + 1] = as_u(__floats2half2_rn(wb0, wb1));
                }
                tmem_st32p(lanes + 32 * c, st);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.pfull);
            if (w == 0) {
                if (!(ok = mbar_wait_warp(&S.abort, &S.vfull, now & 1u, P.status, 72) && mbar_wait_warp(&S.abort, &S.pfull, now & 1u, P.status, 73))) break;
                tc_fence_after();
                const unsigned long long vd = smem_desc(smem_u32(S.v), 128 * 128, 1024, 2);
#pragma unroll
                for (int k = 0; k < 8; ++k)                  // sixteen tokens: two groups of eight rows
                    umma_f16_ts(tmem + O_COL, tmem + 8 * k, vd + (unsigned)((k * 2048) >> 4), ID_O, i > 0 || k > 0);
                umma_commit(&S.vfree);
            }
            if (i + 1 < n) {
                const unsigned char* ahead;
                keys(i + 1);
                ahead = block;
                if (w == 0 && !(ok = scores(i + 1))) break;
                if (!(ok = mbar_wait_warp(&S.abort, &S.vfree, now & 1u, P.status, 75))) break;
                values(i + 1, ahead);
            }
        }
        // ---- the rows' sums, by way of shared memory ----
        if (ok && mbar_wait_warp(&S.abort, &S.vfree, (it + n - 1) & 1u, P.status, 77)) {
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
                unsigned r[32];
                tmem_ld64(lanes + O_COL + 64 * c, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int col = 64 * c + 8 * j + c0;
                    *reinterpret_cast<uint2*>(S.k + sum_at(r0, col >> 2) + 4 * (col & 3)) = make_uint2(r[4 * j], r[4 * j + 1]);
                    *reinterpret_cast<uint2*>(S.k + sum_at(r0 + 8, col >> 2) + 4 * (col & 3)) = make_uint2(r[4 * j + 2], r[4 * j + 3]);
                }
            }
        }
        {
            const auto sum4 = [&](f32x2 v) {
                unsigned u0, u1;
                unpk(v, u0, u1);
                float t = __uint_as_float(u0) + __uint_as_float(u1);
                t += __shfl_xor_sync(0xffffffffu, t, 1);
                return t + __shfl_xor_sync(0xffffffffu, t, 2);
            };
            const float ta = sum4(la), tb = sum4(lb), xa = sum4(ea), xb = sum4(eb);
            if ((lane & 3) == 0) {
                S.l[r0] = ta;
                S.l[r0 + 8] = tb;
                S.add[r0] = xa;
                S.add[r0 + 8] = xb;
                S.m[r0] = Ma;
                S.m[r0 + 8] = Mb;
            }
        }
        tc_fence_before();
        it += n;
        __syncthreads();
        tc_fence_after();
        const bool starts = piece.starts, ends = piece.ends;
        if (S.abort) break;
        {
            float* sums = P.parts + ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * PART;
#pragma unroll 1
            for (int q0 = 0; q0 < ROWS; q0 += 32) {
                const int row = q0 + (tid >> 3), l8 = tid & 7;
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
                        *reinterpret_cast<float4*>(sums + row * 128 + 64 * (q >> 1) + 8 * l8 + 4 * (q & 1)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                    if (l8 == 0) {                           // the sums and the totals go by the same M: 64 times their size
                        sums[ROWS * 128 + row] = m;
                        sums[ROWS * 128 + ROWS + row] = total;
                        sums[ROWS * 128 + 2 * ROWS + row] = extra;
                        sums[ROWS * 128 + 3 * ROWS + row] = m + 6.f;
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
    if (w == 0) {
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
