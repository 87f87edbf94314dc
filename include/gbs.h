/*
 * gbs.h -- C ABI of the B200 (sm_100a) rotate-and-quantize library.
 *
 * The library implements the online activation / KV path of "Gradual Binary Search and
 * Dimension Expansion" (arXiv 2504.13989): every token row of width d is zero-padded to
 * d' = m * 2^k (Section 4.2, Eq. (2)), rotated by the normalised Hadamard matrix
 * H_{d'} = H_m (x) H_{2^k} / sqrt(d')  (Sylvester recursion of Eq. (1) for the power of two,
 * Paley's Algorithm 2 for the factor m, 1/sqrt(n) normalisation of Appendix A), quantized per
 * token or per group with the symmetric uniform quantizer of Section 2.1 under the clip ratio
 * alpha of Section 3.1, and bit-packed.  A companion call scores K candidate clip ratios by
 * quantization error, the quantity a clip-ratio search such as Algorithm 1 queries.
 *
 * Conventions
 *   - Every function returns an int status: GBS_OK (0) or a negative GBS_ERR_* code.
 *     Nothing throws, prints, or synchronises the device.  Argument errors are detected on
 *     the host before any kernel is launched; no call can fault the device through a bad
 *     size (pointers themselves cannot be validated and are the caller's responsibility).
 *   - "device pointer" = memory of the CUDA device that was current when the plan was
 *     created.  The caller owns all buffers; the library never allocates per call.
 *   - Work is enqueued on the CUDA stream passed as `cuda_stream` (a cudaStream_t cast to
 *     void*; NULL = the legacy default stream) and the call returns without waiting.
 *   - Rotated coordinate i of a row is i = a * 2^k + c with a in [0,m), c in [0,2^k):
 *     y[i] = (1/sqrt(d')) * sum_{a',c'} H_m[a,a'] * (-1)^popcount(c & c') * x_pad[a'*2^k + c'].
 *   - Quantizer: per token (group = 0) or per run of `group` consecutive rotated coordinates,
 *     M = max|y|, Delta = alpha * M / D with D = 2^(bits-1) - 1, code q = clamp(rint(y/Delta),
 *     -D, D) (round half to even); M = 0 gives codes 0 and Delta 0.  (Read with `bits` as the
 *     number of magnitude bits, this is the printed formula Delta = max|X| / (2^b - 1): the
 *     printed formula at b equals this one at bits = b + 1.)
 *   - Packed codes: element j of a row occupies bits [j*bits, (j+1)*bits) of the row's
 *     little-endian bit stream and holds the low `bits` bits of the two's-complement code
 *     (bits = 4: even index in the low nibble).  Row r starts at byte r * d' * bits / 8.
 *   - Scales: fp32 Delta, layout [n_rows, scales_per_row], scales_per_row = group ? d'/group : 1.
 */
#ifndef GBS_H_
#define GBS_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define GBS_OK 0
#define GBS_ERR_INVALID_ARG (-1) /* a size, pointer or parameter is out of its documented range */
#define GBS_ERR_UNSUPPORTED (-2) /* no Hadamard construction for this m, or d' too large */
#define GBS_ERR_ALIGNMENT (-3)   /* a pointer or stride violates the stated alignment */
#define GBS_ERR_CUDA (-4)        /* a CUDA runtime call failed (e.g. no device, launch error) */
#define GBS_ERR_ALLOC (-5)       /* host or device allocation for the plan failed */

/* element types of activation inputs / dequantized outputs */
#define GBS_DTYPE_F32 0
#define GBS_DTYPE_BF16 1

/* gbs_plan_create_ex flags */
#define GBS_PLAN_ASYMMETRIC 1    /* asymmetric quantizer (KV entries, Section 5.1): see gbs_plan_create_ex */

/* gbs_dequantize flags */
#define GBS_INVERSE_ROTATE 1

/* largest padded width and largest number of clip-ratio candidates per call */
#define GBS_MAX_D_PAD 32768
#define GBS_MAX_CANDIDATES 64
/* largest padded width gbs_rotate_quantize_static serves from its fixed device array */
#define GBS_STATIC_MAX_D_PAD 4096

typedef struct gbs_plan gbs_plan_t;

typedef struct gbs_plan_info {
    int d, d_pad, m, k;            /* d' = m * 2^k                                   */
    int bits, group;               /* group = 0: one scale per token                  */
    float alpha;
    int levels;                    /* D = 2^(bits-1) - 1; codes lie in [-D, D]        */
    int q_lo, q_hi;                /* -D, +D                                          */
    int64_t code_bytes_per_row;    /* d' * bits / 8                                   */
    int scales_per_row;            /* group ? d'/group : 1                            */
    int asymmetric;                /* 1 for a GBS_PLAN_ASYMMETRIC plan                */
    int scale_floats_per_row;      /* scales_per_row, or 2 * scales_per_row when asymmetric */
    int variant;                   /* kernel family chosen for bf16 rows: 0 = generic shared-memory path,
                                      1 = tensor-core path for d' = 32 * U with 16 <= U = m * 2^j <= 128,
                                      d % 32 == 0 and group in {0, 32 .. 1024}, 2 = tensor-core path for
                                      d' = 128 rows (m = 1, group in {0, 32, 64, 128}), 3 = tensor-core path for
                                      4096 < d' = 32 * G * U <= 32768 (G in {2, 4, 8}, U as above, d a multiple of
                                      32 * G, group 0 or 32 .. 1024 * G; two kernels: one sweep for G = 2 with
                                      group 0 or 128 .. 2048, three otherwise), 4 = dense tensor-core contraction with the full
                                      Paley matrix (d' = m), 5 = as 3 where also d' = 128 * U with 80 <= U <= 256,
                                      d % 128 == 0 and group <= 4096: rotate-quantize keeps the rest of the transform
                                      in registers, clip scoring runs as in 3 (GBS_NO_UVR=1 forces 3) (set GBS_FORCE_GENERIC=1 in the
                                      environment before gbs_plan_create to force 0; GBS_NO_PDL=1: its launches,
                                      plain dequantize and KV restore among them, without programmatic
                                      stream serialization) */
} gbs_plan_info_t;

/*
 * Create a plan (Section 4.2 for d -> d'; Eq. (1) and Algorithm 2 for the rotation;
 * Section 2.1 / 3.1 for bits and alpha).
 *   d       row width, 1 <= d <= d_pad
 *   d_pad   d' = m * 2^k with 2^k >= 8 and d' <= GBS_MAX_D_PAD
 *   m       1 (pure Sylvester); 12, 20, 24, 44, 48, 60, 68, 72, 80, 84, 104 or 108 (Algorithm 2 with the
 *           prime p = m-1 = 3 mod 4); or 28 (Algorithm 2 over GF(27) = GF(3)[x]/(x^3+2x+1), elements
 *           indexed c0 + 3 c1 + 9 c2).  Other orders return GBS_ERR_UNSUPPORTED.
 *           Full orders: d_pad = m (2^k = 1) is accepted when m - 1 is a prime = 3 mod 4, m a multiple of 8 and
 *           128 <= m <= 4096 -- the rotation is then the Paley matrix H_m itself, e.g. d = 1536, d_pad = m = 1544
 *           (Section 5.2.2).  Such plans take bf16 rows with d a multiple of 8 and group = 0, run as a dense
 *           tensor-core contraction, and support gbs_rotate_quantize and gbs_dequantize (both forms; the inverse
 *           rotation is a dense contraction too); gbs_clip_error and the searches return GBS_ERR_UNSUPPORTED
 *           for them.
 *   bits    3 or 4
 *   group   0, or a power of two >= 8 dividing 2^k (so a group never straddles a block of H_m)
 *   alpha   0 < alpha <= 1
 * The plan owns small device tables (the signs of H_m) on the current device, is immutable
 * and may be used from several threads / streams at once.  *out is written only on success.
 */
int gbs_plan_create(gbs_plan_t** out, int d, int d_pad, int m, int bits, int group, float alpha);

/*
 * gbs_plan_create with flags.  flags = 0 is gbs_plan_create.
 * GBS_PLAN_ASYMMETRIC selects the asymmetric uniform quantizer the paper uses for KV entries
 * (Section 5.1 names it, with "a group size of 128", but prints no formula; this is the textbook one,
 * with the clip ratio of Section 3.1 shrinking both ends of the range).  Per token or group:
 *     lo = alpha * min y,  hi = alpha * max y,  Delta = (hi - lo) / (2^bits - 1),
 *     code = clamp(rint((y - lo) / Delta), 0, 2^bits - 1)  (round half to even),  yhat = code * Delta + lo;
 * a constant group gives codes 0 and Delta 0.  Codes are UNSIGNED `bits`-bit fields, packed as usual;
 * `scales` holds the pair (Delta, lo) per group: layout [n_rows, scales_per_row, 2].
 * Limits: d' = 128 rows (m = 1), group 0, 32, 64 or 128, bf16 input; other shapes return
 * GBS_ERR_UNSUPPORTED.  gbs_clip_error and gbs_search_clip_ratio return GBS_ERR_UNSUPPORTED for such a
 * plan; gbs_dequantize (both forms) honours it.
 */
int gbs_plan_create_ex(gbs_plan_t** out, int d, int d_pad, int m, int bits, int group, float alpha, int flags);

/* Free a plan.  NULL is accepted.  Work already enqueued with the plan must have finished. */
int gbs_plan_destroy(gbs_plan_t* plan);

/* Report the derived sizes of a plan. */
int gbs_plan_info(const gbs_plan_t* plan, gbs_plan_info_t* out);

/*
 * Read and clear the plan's device-side status word.  The tensor-core kernels bound every wait on a
 * barrier; if one ever expires the kernel records a non-zero code here, frees what it holds and
 * returns instead of hanging (the results of that launch are then invalid).  0 = no such event.
 * This call copies 4 bytes from the device and therefore WAITS for the device's pending work.
 * (Not an operation of the paper: a diagnostic of this implementation.)
 */
int gbs_plan_device_status(const gbs_plan_t* plan, int* out);

/*
 * Self-test of the bounded waits (a diagnostic of this implementation, not an operation of the paper): one
 * thread of a one-block kernel on the current device waits, for at most `limit_us` microseconds (1 .. 1 000 000),
 * on a barrier that nothing arrives at.  The wait must run out: the call then returns GBS_OK with *code_out = 7
 * (the code that wait records in its status word), *abort_out = 1 (the flag it raises for the other roles of a
 * kernel) and *waited_us_out = how long it waited (limit_us plus at most a few polling periods).  Nothing
 * faults or hangs; the context stays usable.  Runs on the default stream and WAITS for the device.
 */
int gbs_selftest_wait_expiry(int limit_us, int* code_out, int* abort_out, int* waited_us_out);

/*
 * Fused pad -> rotate -> per-token/group absmax -> scale -> round/clip -> pack
 * (Section 4.2, Eq. (1), Algorithm 2, Section 2.1, Section 3.1), one pass over x.
 *   x            device, n_rows rows of d elements of x_dtype; row r starts at element
 *                r * x_row_stride.  Must be 16-byte aligned with x_row_stride * sizeof(elem)
 *                a multiple of 16, x_row_stride >= d.
 *   codes        device, n_rows * d' * bits / 8 bytes, 16-byte aligned
 *   scales       device, n_rows * scale_floats_per_row floats (scales_per_row Deltas per row; (Delta, lo)
 *                pairs for an asymmetric plan)
 *   y_opt        NULL, or device n_rows * d' floats receiving the rotated normalised values
 *                (16-byte aligned)
 * n_rows = 0 is a successful no-op.
 */
int gbs_rotate_quantize(const gbs_plan_t* plan, const void* x, int x_dtype, int64_t n_rows,
                        int64_t x_row_stride, void* codes, float* scales, float* y_opt,
                        void* cuda_stream);

/*
 * gbs_rotate_quantize for callers that must not allocate device memory.  (The paper has no counterpart
 * of this call; it exists for the deployment reasons below.)
 *
 * A plan owns a little device memory that gbs_plan_create obtains from cudaMalloc: the tensor-core
 * kernel reads a 32 KB table (the +-1 matrix H_m (x) H_{2^j} laid out for the MMA unit) and has a
 * status word.  Some callers cannot go through that: a serving process whose memory pool has already
 * claimed all of the GPU, so that a later cudaMalloc fails; a real-time loop that may not take the
 * device-wide synchronisation cudaMalloc and cudaFree imply; code that is handed a device it may use
 * but not grow on.  For them this call takes the plan's parameters directly and keeps the table and
 * the status word in one fixed array inside the library's device image (about 32 KB on every GPU
 * that loads the library, held until the process exits).  It calls no cudaMalloc, cudaFree or other
 * allocating routine, and the caller still passes the input and both outputs.
 *
 *   d, d_pad, m, bits, group, alpha   as for gbs_plan_create, with these extra limits: bf16 rows only;
 *                d_pad <= GBS_STATIC_MAX_D_PAD; m one of 1, 12, 20, 24, 28 (the array's writer keeps one
 *                32-bit sign word per row of H_m); d_pad and d multiples of 32; d_pad / 32 a multiple of
 *                16; group 0 or 32 .. 1024.  Anything else in gbs_plan_create's range returns
 *                GBS_ERR_UNSUPPORTED ("larger than the fixed array serves, or outside its kernel"):
 *                use a plan for those.
 *   x, n_rows, x_row_stride, codes, scales, cuda_stream   as for gbs_rotate_quantize with
 *                x_dtype = GBS_DTYPE_BF16; results are identical to the plan-based call.
 *
 * The array is shared by every call on a device and keeps what the last call left in it:
 *   - The first call on a device looks up the array's device address (with that device current).  Make
 *     that first call before any stream capture begins.  The status word starts at zero (the array is
 *     zero-initialised when the library's device code is loaded).
 *   - A call reuses the table as it stands only if the previous call on that device used the same
 *     (d_pad, m) on the same stream; every other call first rewrites the table with a small kernel on
 *     `cuda_stream`, so its own kernel is ordered behind the write.  A call made while `cuda_stream` is
 *     being captured always includes the rewrite, and after the first captured call on a device every
 *     call rewrites (a replay changes the array without passing through this function).
 *   - Calls that can overlap on the GPU (different streams, or different host threads without
 *     ordering between their streams) are safe when they all use the same (d_pad, m): they rewrite the
 *     same bytes.  Overlapping calls with DIFFERENT (d_pad, m) race on the array: serialise them, or
 *     give the concurrent users plans.
 */
int gbs_rotate_quantize_static(int d, int d_pad, int m, int bits, int group, float alpha, const void* x,
                               int64_t n_rows, int64_t x_row_stride, void* codes, float* scales,
                               void* cuda_stream);

/*
 * Read and clear the status word of gbs_rotate_quantize_static on the current device (the counterpart of
 * gbs_plan_device_status for the plan-free call: 0 = no bounded wait has expired since the last read).
 * Copies 4 bytes from the fixed array, so it WAITS for the device's pending work; allocates nothing.
 * (The paper has no counterpart of this call: a diagnostic of this implementation.)
 */
int gbs_static_device_status(int* out);

/*
 * Inverse of the quantizer: yhat = q * Delta (Section 2.1) in the rotated domain, width d';
 * with GBS_INVERSE_ROTATE also xhat = (H_{d'}^T yhat / sqrt(d'))[0:d] (rotations are undone by
 * the transpose, Section 2.3.1), width d.
 *   codes, scales  device, layouts as written by gbs_rotate_quantize
 *   out            device, n_rows * (d' or d) elements of out_dtype, rows contiguous,
 *                  16-byte aligned
 * The inverse rotation of symmetric plans with d' = 32 U (d a multiple of 32) or, beyond 4096, d' = 64 U (d a multiple of
 * 64), 16 <= U <= 128, and one scale per token or per group of at least 32 or 64 runs on the tensor cores; with one scale
 * the integer codes are rotated exactly and multiplied by Delta / sqrt(d') once at the end, with groups the operand
 * q * Delta is held to 22 bits below the token's largest scale.  Where m = 1, d' <= 2048 and the plan has groups, a
 * general kernel takes widths and numbers of rows at which it is faster; a row's result may then differ in the last fp32
 * bits with the number of rows.  d' = 128 rows with one scale or (Delta, lo) pair per row are rotated exactly in
 * registers.
 */
int gbs_dequantize(const gbs_plan_t* plan, const void* codes, const float* scales, int64_t n_rows,
                   void* out, int out_dtype, int flags, void* cuda_stream);

/*
 * Score K clip ratios: for each alpha_k, err_sum[k] += sum over rows and rotated coordinates of
 * (y - yhat_k)^2, yhat_k being the quantizer output (Section 2.1) under clip ratio alpha_k
 * (Section 3.1).  The plan's own alpha is ignored; bits and group are honoured.
 *   x, x_dtype, n_rows, x_row_stride   as for gbs_rotate_quantize
 *   alphas_host   HOST pointer to K floats, each in (0, 1]; copied at call time
 *   K             1 .. GBS_MAX_CANDIDATES
 *   err_sum       device, K doubles, ACCUMULATED into (the caller zeroes them)
 *   err_rows_opt  NULL, or device n_rows * K floats receiving the per-row sums
 * Which kernel scores a call depends on its shape, its list and whether per-row sums are asked for: one histogram for all
 * candidates (d' <= 4096, group 0 or 128 and more, bf16) or a pass per eight.  The histogram rounds each
 * residual to at most 1.5 x 2^-23 max|y| (of the token or group), the passes round each candidate's Delta to 2^-24 of itself, so one alpha's sum from two
 * calls agrees to about 2e-7 of the sum where the rows are ordinary, and to 1.5 x 2^-22 max|y| sqrt(n err) where the candidate fits n values almost
 * exactly (2e-5 of the sum where they are a thousandth off); a search that compares sums from different calls decides closer ties by chance.
 */
int gbs_clip_error(const gbs_plan_t* plan, const void* x, int x_dtype, int64_t n_rows,
                   int64_t x_row_stride, const float* alphas_host, int K, double* err_sum,
                   float* err_rows_opt, void* cuda_stream);

/*
 * Result of gbs_search_clip_ratio (host memory).
 */
typedef struct gbs_search_result {
    float alpha;        /* the clip ratio kept at the end (m of Algorithm 1)                       */
    float a, b;         /* the final bracket, b - a <= eps                                          */
    double err;         /* the objective at alpha: sum over rows and coordinates of (y - yhat)^2   */
    int iterations;     /* passes through the loop body of Algorithm 1                              */
    int evaluations;    /* objective values the algorithm consumed: iterations + 1                  */
    int rounds;         /* gbs_clip_error launches used to obtain them                              */
} gbs_search_result_t;

/*
 * The bracket search of Algorithm 1 (Gradual Binary Search, the loop for one projection) for the clip
 * ratio of the rows in x, with the quantization error of gbs_clip_error as the objective (the paper
 * minimises perplexity; this library has no model to evaluate, Sections 3.1 and 4.1).
 * Start a = 0, b = 1, m = 1/2; on even iterations probe (a+m)/2, on odd ones (b+m)/2; a probe that
 * lowers the objective becomes the new m and halves the bracket towards it, otherwise the bracket end
 * on the probe's side moves to the probe; stop when b - a <= eps.  The states visited are those of the
 * algorithm as printed; evaluations are grouped: each round scores the probes of the next five
 * iterations' decision tree (at most 31 clip ratios) in one gbs_clip_error launch.
 *   x, x_dtype, n_rows, x_row_stride   as for gbs_clip_error (n_rows >= 1)
 *   eps        0 < eps < 1 (1/64 gives 9 to 13 iterations)
 *   work_dev   device, GBS_MAX_CANDIDATES doubles, 8-byte aligned, overwritten
 *   out_host   host, written on success
 * BLOCKS: after every round the call waits for `cuda_stream` to read the K sums back.
 */
int gbs_search_clip_ratio(const gbs_plan_t* plan, const void* x, int x_dtype, int64_t n_rows,
                          int64_t x_row_stride, float eps, double* work_dev, gbs_search_result_t* out_host,
                          void* cuda_stream);

/*
 * Weight side of the expansion (Section 4.2, Eq. (2)): the rows of W (one per output channel, width d) are
 * zero-padded to d', rotated by the same H_{d'} / sqrt(d') as the activations and quantized round-to-nearest with
 * the plan's bits, group and alpha -- exactly gbs_rotate_quantize applied to the rows of W, which is what makes
 * (H x_pad)^T (H w_pad) / d' = x^T w hold code for code.  With group = 0 there is one scale per output channel, the
 * form gbs_quantized_matmul consumes.  Done once, offline.
 *   w, w_dtype, n_out, w_row_stride   the weight matrix [n_out, d] (device), as x / x_dtype / n_rows / x_row_stride
 *   codes, scales                     as for gbs_rotate_quantize
 */
int gbs_weight_rotate_quantize(const gbs_plan_t* plan, const void* w, int w_dtype, int64_t n_out, int64_t w_row_stride,
                               void* codes, float* scales, void* cuda_stream);

/*
 * The layer's output straight from the packed codes of both sides (Eq. (2); Section 2.3.1 on keeping the inverse
 * rotation out of the online path): out[t][o] = Delta_x[t] * Delta_w[o] * sum_j q_x[t][j] * q_w[o][j], j over the
 * d' rotated coordinates -- the product of the dequantized rotated activation and the dequantized rotated weight,
 * which equals x^T w up to the two quantization errors.  The sum is an int8 x int8 -> int32 contraction on the
 * tensor cores (exact); the rotated activation is never materialised as floats.
 *   plan_x, codes_x, scales_x, n_tokens   activations as written by gbs_rotate_quantize
 *   plan_w, codes_w, scales_w, n_out      weights as written by gbs_weight_rotate_quantize
 *   out, out_dtype, out_row_stride        device, [n_tokens, n_out] fp32 or bf16, row stride in elements (>= n_out),
 *                                         any alignment of its type
 * Limits: both plans on one device with the same d, d' and m, symmetric, group 0 (one scale per token and per
 * output channel, so the scales leave the sum), d' a multiple of 128; bits may differ (3 or 4 each).  Other plans
 * return GBS_ERR_UNSUPPORTED.
 */
int gbs_quantized_matmul(const gbs_plan_t* plan_x, const void* codes_x, const float* scales_x, int64_t n_tokens,
                         const gbs_plan_t* plan_w, const void* codes_w, const float* scales_w, int64_t n_out,
                         void* out, int out_dtype, int64_t out_row_stride, void* cuda_stream);

/*
 * ------------------------------------------------------------------------------------------------------------------
 * Paged KV cache in four bits, and attention over it (Section 5: the cache holds rotated, quantized rows; Section 2.3.1: a
 * rotation that both sides of a product share leaves it unchanged, so keys and values stay rotated and only the query and
 * the result are turned).  The paper has no counterpart of the paging.
 *
 * Plans: bits 4, d' = 128 (m = 1), group 0 or 128, d a multiple of 8, symmetric or asymmetric; other plans return
 * GBS_ERR_UNSUPPORTED.  d is the width of a head; narrower heads are zero-padded to 128 coordinates (Section 4.2).
 *
 * Pool: `pages` holds n_pages pages of gbs_kv_page_bytes bytes.  A page holds, for each KV head in turn, a block of
 * page_size tokens: key codes [page_size][64 bytes], value codes [page_size][64 bytes], key scales and value scales
 * [page_size] floats each (Delta), or [page_size][2] for an asymmetric plan (Delta, lo).  Codes are packed as everywhere.
 * page_table [n_seqs][max_pages] lists the pages of each sequence in order; only the first ceil(lengths[s] / page_size) entries
 * of a row are read, the others count for nothing.  lengths [n_seqs]: tokens of each sequence.  refs [n_pages]: how many
 * sequences hold a page; 0 = free.  A page that is not full belongs to one sequence alone.  A new pool has lengths
 * and refs 0; no other preparation is needed.  All five arrays are device memory and belong to the caller.
 *
 * A call's items are sequences: item i is sequence seqs[i], or i where seqs is NULL (device int32).  Its tokens are rows
 * cu_tokens[i] .. cu_tokens[i + 1] - 1 of the call's row tensors (device int32, n_items + 1 values that do not fall, from 0), or row i
 * alone where cu_tokens is NULL.  They are the LAST tokens of the sequence as lengths[] has it: a step extends the
 * sequences first, then appends and attends.  So an item that gbs_kv_extend refused must not be appended: its rows would replace the
 * sequence's last ones, which other sequences may share; gbs_kv_append_extended leaves such items out.  Rows behind
 * cu_tokens[n_items] count for nothing and are not written.
 * Numbers that only the device knows are checked there: an item whose sequence is out of range, a token whose position is
 * below 0 or whose page is not one of the pool's is left out (a row that would be written from it becomes 0).
 *
 * Calls are enqueued on `cuda_stream` and may be captured.  Calls that change a pool and calls that use it have to be ordered
 * by the caller, as any use of one buffer from two streams.
 */
#define GBS_KV_MAX_ITEMS 8192

typedef struct gbs_kv_cache {
    void* pages;            /* 16-byte aligned */
    int64_t n_pages;        /* 1 .. 2^30 */
    int n_kv_heads;         /* 1 .. 1024 */
    int page_size;          /* 16, 32, 64 or 128 tokens */
    int32_t* page_table;
    int32_t* lengths;
    int32_t* refs;
    int n_seqs, max_pages;  /* n_seqs * max_pages entries; max_pages at most 2^20 */
} gbs_kv_cache_t;

/* what became of an item of gbs_kv_extend, gbs_kv_fork and gbs_kv_evict (device int32) */
#define GBS_KV_DONE 0
#define GBS_KV_BAD_INDEX 1    /* a sequence out of range, or a negative count */
#define GBS_KV_NOT_EMPTY 2    /* the target of a fork holds tokens */
#define GBS_KV_NO_PAGES 3     /* not enough free pages for this item and those before it */
#define GBS_KV_TOO_LONG 4     /* the sequence would not fit its row of the table */
#define GBS_KV_DUPLICATE 5    /* an earlier item of the call names the same sequence (the same target) */

/* Bytes of one page: n_kv_heads * page_size * (128 + 8 * scale floats of a row).  Host only. */
int gbs_kv_page_bytes(const gbs_plan_t* plan, int n_kv_heads, int page_size, int64_t* out);

/*
 * Room for counts[i] more tokens in sequence seqs[i]: lengths grow, and free pages enter the table, the lowest free ones first,
 * to the items in their order.  An item that is refused (status_out[i] != GBS_KV_DONE) leaves its sequence and the pool's refs as they
 * were; from the first one that the free pages do not suffice for, every item that needs a page is refused.
 *   seqs, counts   device int32 [n_items], n_items 0 .. GBS_KV_MAX_ITEMS; seqs NULL: sequence i; counts NULL: one token each
 *   status_out     device int32 [n_items]
 */
int gbs_kv_extend(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* counts, int n_items,
                  int32_t* status_out, void* cuda_stream);

/*
 * Sequence dst[i], which has to be empty, becomes a copy of sequence src[i]: full pages are shared (refs + 1), the tokens of a last
 * page that is not full are copied into a page of its own, taken as by gbs_kv_extend.  All pairs see the
 * sequences as they were before the call; one source may have any number of targets.
 *   src, dst, status_out   device int32 [n_items], n_items 0 .. GBS_KV_MAX_ITEMS
 */
int gbs_kv_fork(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* src, const int32_t* dst, int n_items,
                int32_t* status_out, void* cuda_stream);

/*
 * The sequences end: their lengths become 0, refs of their pages fall by 1, and pages at 0 are free.  A sequence out of range
 * is left out; one that is named twice ends once.  Page contents and table entries stay.
 */
int gbs_kv_free(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, int n_items, void* cuda_stream);

/*
 * Move the pages in use (refs > 0) of `cache` into pages 0, 1, .. of `into`, in the order of their numbers, and write `into`'s table
 * (entries behind a sequence's last page become -1), lengths and refs.  `into` is another pool of the same n_kv_heads,
 * page_size, n_seqs and max_pages with any number of pages, none of its arrays shared with `cache`; what it held is lost.
 *   page_map    device int32 [cache->n_pages], receives each page's new number, -1 for a free one
 *   n_live      device int32, receives the number of pages in use.  If it exceeds into->n_pages, the pages beyond that are not
 *               moved and stand as -1 in page_map and in the table: such an `into` is not to be used.
 */
int gbs_kv_compact(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const gbs_kv_cache_t* into, int32_t* page_map,
                   int32_t* n_live, void* cuda_stream);

/*
 * gbs_rotate_quantize of key and value rows, written into the pages of their tokens.
 *   k, v              device bf16 [n_tokens][n_kv_heads][d], rows 16-byte aligned: token t, head h starts at element
 *                     t * token_stride + h * head_stride, strides multiples of 8 (k and v have the same)
 *   n_tokens          rows that k and v hold; cu_tokens NULL: n_tokens = n_items
 * Where two items name one sequence, both write its last tokens, and either's bytes may stay.
 * A row that holds a NaN gets a scale that is one: attention over it, and what is read back, are NaN.
 *
 * gbs_kv_append_extended writes the rows of those items alone that gbs_kv_extend has served, so that a step which is enqueued as a whole,
 * or captured, may run out of pages: rows of an item with status[i] != GBS_KV_DONE are left out.
 *   status            device int32 [n_items], as gbs_kv_extend wrote it for the same items; NULL: all items are written
 */
int gbs_kv_append(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                  int64_t n_tokens, const void* k, const void* v, int64_t token_stride, int64_t head_stride, void* cuda_stream);
int gbs_kv_append_extended(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                           int64_t n_tokens, const void* k, const void* v, int64_t token_stride, int64_t head_stride, const int32_t* status,
                           void* cuda_stream);

/*
 * The rows that the cache stands for, back in their own basis: gbs_dequantize with GBS_INVERSE_ROTATE of the items' tokens.
 *   k_out, v_out      device bf16 [n_tokens][n_kv_heads][d], contiguous, 16-byte aligned
 */
int gbs_kv_read(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                int64_t n_tokens, void* k_out, void* v_out, void* cuda_stream);

/* gbs_kv_attention flags */
#define GBS_KV_CAUSAL 1       /* a token sees the cache up to its own position; without it, all of its sequence, of which it need not be a part */

/*
 * Attention of the items' query tokens over the cache: with khat, vhat the rows that the cache stands for,
 *     out[t][h] = sum_j p_j vhat_j,   p = softmax over the visible j of (scale * q[t][h] . khat_j),
 * KV head h / (n_heads / n_kv_heads) serving query head h.  Token t at position p of its sequence sees positions j <= p (causal) and,
 * with window > 0, j > p - window.  A row that sees nothing becomes 0.
 *   q, out            device bf16, [n_tokens][n_heads][d] with strides in elements as in gbs_kv_append; out's own strides.  No row of
 *                     out overlaps another one or a row of q
 *   n_heads           a multiple of n_kv_heads, at most 1024 query heads per KV head
 *   max_tokens        no item has more tokens (1 where cu_tokens is NULL); what is beyond it is left as it is.  It chooses the
 *                     kernel and bounds what is looked through for work, so the closer the better.
 *                     n_items * max_tokens * query heads of a KV head: at most 2^28
 *   max_len           about the length of the call's longest sequence (0: the table's width).  It chooses how far the work is split, never
 *                     what is read: a longer sequence is read whole, if more slowly.
 *   scale             0: 1 / sqrt(d)
 *   workspace         device, gbs_kv_attention_workspace bytes, 16-byte aligned; overwritten, needs no preparation, and one call at
 *                     a time may use it
 * Up to 16 rows a KV head and item, rotated query rows are rounded to 16 bits of their largest coordinate, and codes enter as they are; with more
 * rows query coordinates, scales and the cached coordinates that they give are each rounded to 11 bits.  Probabilities are rounded to
 * 11 bits; sums and softmax statistics are fp32.  With more than 16 rows, a row more than 2^21 smaller than another of the same 32 tokens
 * (positions 32 i .. 32 i + 31) has fewer bits, and value rows more than 2^100 smaller than others that
 * the same row sees may lose their share of the softmax's sum.  A token with a scale that is infinite or a NaN makes the rows that see
 * it NaN.
 */
int gbs_kv_attention_workspace(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, int n_heads, int64_t n_tokens, int max_tokens,
                               int64_t* bytes_out);
int gbs_kv_attention(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                     int64_t n_tokens, int max_tokens, int max_len, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                     int n_heads, float scale, int window, int flags, void* out, int64_t out_token_stride, int64_t out_head_stride,
                     void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * The same attention for items whose sequences begin alike, as forks of one prompt do: what a group's sequences have in common is read
 * once for all of the group's rows, where that is likely to take less time.  Common are the full pages, from a sequence's first on, that stand in the page
 * tables of all items of the group that have tokens and lie before the tokens of each of them; the call finds them in the tables, so a group of
 * sequences that share nothing is attended over as well.  Results differ from gbs_kv_attention's by rounding alone.  There is no window: what a window leaves of a
 * common prefix differs from item to item.
 *   groups            device int32 [n_groups + 1], values that do not fall: group g is items groups[g] .. groups[g + 1] - 1, and items of no
 *                     group share nothing.  NULL: all items are one group (n_groups is 1)
 *   n_groups          1 .. GBS_KV_MAX_ITEMS
 *   max_own           about the most tokens that a sequence has behind what its group shares (0: the table's width), as max_len of gbs_kv_attention
 *   max_prefix        about the most tokens that a group shares (0: the table's width, which a table with room to spare makes too much).  By it and the sizes it is
 *                     judged whether sharing gains anything: finding the groups and joining what their rows got costs some 20 to 45 microseconds, also where they turn
 *                     out to share little or nothing.  Where it is not likely to gain more, the call reads as gbs_kv_attention does
 *   n_tokens          query heads of a KV head * n_tokens: at most 2^28, and so query heads of a KV head * n_items * max_tokens, as in gbs_kv_attention
 *   workspace         gbs_kv_shared_attention_workspace bytes, 16-byte aligned, overwritten and used by one call at a time; 528 bytes a token and query head where prefixes are shared.  The same
 *                     number of items, tokens and groups and the same max_tokens and max_prefix as in the call
 * Precision is gbs_kv_attention's, but that with many rows a cached coordinate is rounded once, to 11 bits; rows of a prefix count as many rows (more than 16) where groups have more than 32 rows a KV head on average.
 */
int gbs_kv_shared_attention_workspace(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, int n_items, int64_t n_tokens, int max_tokens,
                                      int n_groups, int max_prefix, int n_heads, int64_t* bytes_out);
int gbs_kv_shared_attention(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                            int64_t n_tokens, int max_tokens, const int32_t* groups, int n_groups, int max_own, int max_prefix, const void* q,
                            int64_t q_token_stride, int64_t q_head_stride, int n_heads, float scale, int flags, void* out,
                            int64_t out_token_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * The softmax weight that each cached token gets from the items' query tokens, by KV head: with p the probabilities of gbs_kv_attention for these
 * arguments and j a position of item i's sequence s,
 *     mass[s][kv head][j] = decay * base[s][kv head][j] + sum of p_j over the item's query tokens and the query heads of the KV head,
 * where base counts as 0 for the item's own tokens, which had no weight before this call.  Written are positions 0 .. lengths[s] - 1, as far as they lie
 * below `width`, of the sequences of items that have tokens; nothing else is.  Where two items name one sequence, either's sums may stay,
 * where base is mass itself also with the other's as base.
 *   mass, base        device float [n_seqs][n_kv_heads][width]; base is mass itself or does not overlap it, and is not read (NULL will do) where decay is 0
 *   max_tokens        no item has more tokens; what is beyond it gives no weight.  query heads of a KV head * n_tokens: at most 2^28,
 *                     and so query heads of a KV head * n_items * max_tokens
 *   workspace         device, gbs_kv_attention_mass_workspace bytes for the same sizes, 16-byte aligned; overwritten, needs no preparation, and one call at a
 *                     time may use it.  With up to 32 query rows a KV head and item it has room for their scores, 4 bytes a row and position below the width,
 *                     as long as that is 256 MB at most; with more, 532 bytes a token and query head and at most 64 MB for sums
 * Weights belong to positions.  The caller clears those of a sequence that begins anew and copies them for a fork: only the items' own tokens start from 0, and tokens that never
 * were an item's own (those of a prompt before the last ones that a call was made for) start from what stands in base.
 * Scores are right to fp32: query rows are rounded to 24 bits of their largest coordinate, its sign among them, codes enter as they are, sums of products are exact, and
 * what they become is rounded as a float.  With more than 32 query rows a KV head and item it is 23 bits, and the logarithm of a row's sum is rounded as well, so that all
 * of a row's weights may be off by 2^-24 of its largest score's size (in units of log 2).  Scores beyond 2^24 have no units in fp32: weights are finite, and no more.  Value
 * rows count for nothing.  A token whose key scale is infinite or a NaN makes the rows that see it, and so what they see, NaN.
 * Where a bounded wait runs out (gbs_plan_device_status), a weight is what it was or what it was to become, nothing else; all are what they were if that
 * is before all rows' sums are known.
 */
int gbs_kv_attention_mass_workspace(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, int n_items, int64_t n_tokens, int max_tokens,
                                    int n_heads, int64_t width, int64_t* bytes_out);
int gbs_kv_attention_mass(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                          int64_t n_tokens, int max_tokens, const void* q, int64_t q_token_stride, int64_t q_head_stride, int n_heads,
                          float scale, int window, int flags, const float* base, float decay, float* mass, int64_t width, void* workspace,
                          int64_t workspace_bytes, void* cuda_stream);

/*
 * Sequences longer than `keep` tokens are cut down to `keep` of them, for each KV head its own: the first `first` ones, the last `recent` ones, and of those between
 * the ones with the largest mass (of two alike the one at the lower position; a NaN counts as the largest, a position from `width` on as 0).  They move to
 * the front of the sequence in their order, into pages of their own, taken as by gbs_kv_extend (so that room for them has to be free, and pages that other sequences
 * share stay as they are); then refs of the pages that the sequence held fall by 1.  A sequence of at most `keep` tokens stays as it is.  Positions are from then on those in what
 * is left: new tokens follow at position `keep`.
 *   keep, recent, first  keep at least 1, recent + first at most keep
 *   mass              device float [n_seqs][n_kv_heads][width], as gbs_kv_attention_mass leaves it
 *   mass_out          the same shape: mass itself, or not overlapping it.  Positions 0 .. of each sequence and KV head receive the mass of the tokens that
 *                     stay (below width); nothing else is written, so that behind them weights of tokens that are gone stand until a call gives new ones their own
 *   kept              device int32 [n_items][n_kv_heads][keep], receives their former positions, which rise; -1 behind the last token of a shorter sequence, and
 *                     in all places of an item that was refused
 *   status_out        device int32 [n_items]; items that are refused (GBS_KV_BAD_INDEX, GBS_KV_DUPLICATE, GBS_KV_NO_PAGES) leave everything as it was
 *   workspace         device, gbs_kv_evict_workspace bytes, 16-byte aligned; overwritten, needs no preparation, and one call at a time may use it
 * A token that stays and whose page is not one of the pool's becomes a row of zeros.
 */
int gbs_kv_evict_workspace(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, int n_items, int keep, int64_t* bytes_out);
int gbs_kv_evict(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, int n_items, int keep, int recent, int first,
                 const float* mass, float* mass_out, int64_t width, int32_t* kept, int32_t* status_out, void* workspace,
                 int64_t workspace_bytes, void* cuda_stream);

/*
 * Self-test of what gbs_kv_attention does when one of its bounded waits runs out (a diagnostic, as gbs_selftest_wait_expiry): the same call,
 * in which the waits of this code in every block's segment of this number (0, 1, ..) count as run out without being made.  The kernel ends, the code
 * stands in the plan's status word, and rows of out may be any numbers; nothing else is written.  A block that has no such wait there
 * ends as always.
 *   code              61 .. 64: up to 16 rows a KV head and item (a unit's copies, a free stage, a free slot for query rows, the query rows);
 *                     71 .. 77: more rows (keys, values, weights, room for keys, room for values, scores, the results)
 */
int gbs_selftest_kv_attention(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens,
                              int n_items, int64_t n_tokens, int max_tokens, int max_len, const void* q, int64_t q_token_stride,
                              int64_t q_head_stride, int n_heads, float scale, int window, int flags, void* out,
                              int64_t out_token_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes, int code,
                              int segment, void* cuda_stream);

/*
 * The same of gbs_kv_shared_attention: in both of its passes, over what groups share and over what is an item's own, where the call has them.
 */
int gbs_selftest_kv_shared_attention(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens,
                                     int n_items, int64_t n_tokens, int max_tokens, const int32_t* groups, int n_groups, int max_own,
                                     int max_prefix, const void* q, int64_t q_token_stride, int64_t q_head_stride, int n_heads,
                                     float scale, int flags, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                     void* workspace, int64_t workspace_bytes, int code, int segment, void* cuda_stream);

/*
 * The same of gbs_kv_attention_mass, whose waits are all in its kernels for more than 32 query rows a KV head and item.
 *   code              81 .. 86: the pass for the rows' sums (scores, room for keys, query rows, keys, room for scores, room for query rows);
 *                     91 .. 99: the pass for the tokens' (keys, query rows, scores, room for keys, keys before their product, query rows before it, room for
 *                     scores, room for query rows, query rows of a tile that no token of a segment is seen by)
 */
int gbs_selftest_kv_attention_mass(const gbs_plan_t* plan, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens,
                                   int n_items, int64_t n_tokens, int max_tokens, const void* q, int64_t q_token_stride,
                                   int64_t q_head_stride, int n_heads, float scale, int window, int flags, const float* base,
                                   float decay, float* mass, int64_t width, void* workspace, int64_t workspace_bytes, int code,
                                   int segment, void* cuda_stream);

/*
 * State of one projection's search (Algorithm 1), a handful of numbers: plain data that may be copied, stored
 * and handed back later to resume the search where it stopped (gbs_search_state_init gives the algorithm's
 * start a = 0, b = 1, m = 1/2).
 */
typedef struct gbs_search_state {
    double a, b, m;     /* the bracket and the kept point                                        */
    double f_m;         /* the objective at m (valid once have_fm is set)                       */
    int iteration;      /* passes through the loop body so far                                   */
    int evaluations;    /* objective values consumed so far                                      */
    int have_fm;        /* f(m) of the start point has been evaluated                            */
    int done;           /* b - a <= eps was reached (set by the search calls)                    */
} gbs_search_state_t;

int gbs_search_state_init(gbs_search_state_t* state);

/*
 * Algorithm 1's loop for one projection with the CALLER's objective, e.g. the perplexity the paper minimises
 * (Sections 3.1, 4.1): f(alpha, ctx) is called once per pass, in the order of the algorithm as printed, plus
 * once for the start point.  Runs until b - a <= eps, or for at most max_iterations passes when that is > 0;
 * `state` (in/out) then resumes.  Host only: touches no device.
 */
typedef double (*gbs_objective_fn)(float alpha, void* ctx);
int gbs_search_clip_ratio_fn(gbs_objective_fn f, void* ctx, float eps, gbs_search_state_t* state,
                             int max_iterations);

/*
 * Algorithm 1's loop for n_tasks projections at once with the quantization error as objective.  The paper walks
 * the projections one after the other because its objective, the model's perplexity, couples them; the
 * quantization error of one projection's input does not depend on the others, so here every round scores the
 * pending probes (the next five iterations' decision tree, at most 31 clip ratios, as in gbs_search_clip_ratio)
 * of EVERY unfinished projection, one gbs_clip_error launch per projection enqueued back to back, and waits once
 * per round.  Each projection visits exactly the states its own gbs_search_clip_ratio call would visit.
 *   tasks       host array: plan, rows (device), dtype, n_rows >= 1 and row stride of each projection; all plans on
 *               one device; n_tasks 1 .. GBS_MAX_SEARCH_TASKS
 *   eps         0 < eps < 1
 *   states      host array, in/out: start from gbs_search_state_init, or resume earlier states
 *   max_rounds  0 = run until every projection is done; otherwise stop after that many rounds (resumable)
 *   work_dev    device, n_tasks * GBS_MAX_CANDIDATES doubles, 8-byte aligned, overwritten
 *   alphas_out  NULL, or host array of n_tasks floats: the list L of Algorithm 1 (the kept point of each projection)
 *   rounds_out  NULL, or the number of rounds this call ran
 * BLOCKS: once per round the call waits for `cuda_stream`.
 */
#define GBS_MAX_SEARCH_TASKS 4096
typedef struct gbs_search_task {
    const gbs_plan_t* plan;
    const void* x;
    int x_dtype;
    int64_t n_rows;
    int64_t x_row_stride;
} gbs_search_task_t;
int gbs_search_clip_ratio_batch(const gbs_search_task_t* tasks, int n_tasks, float eps, gbs_search_state_t* states,
                                int max_rounds, double* work_dev, float* alphas_out, int* rounds_out,
                                void* cuda_stream);

/*
 * Host-only helper: write the m x m sign matrix H_m (row-major, +1 / -1) the plans use
 * (Algorithm 2).  `out_host` must hold m*m bytes.  Needs no device.
 */
int gbs_hadamard_m(int m, int8_t* out_host);

/* Human-readable name of a status code (static string). */
const char* gbs_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* GBS_H_ */
