// Attention over the paged KV cache (gbs_kv_attention): one block per query token and KV head, fp32 throughout.
#include "gbs_kv.cuh"

namespace {

constexpr int THREADS = 128, TILE = 128;

template <bool ASYM>
__global__ __launch_bounds__(THREADS) void k_kv_attn_plain(const __grid_constant__ gbs_kv_attn A)
{
    __shared__ float q[128], p[TILE], add[TILE], red[4];
    __shared__ int item_sh;
    kv_wait_before();
    const int token = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
    if (tid < 32) {
        const int i = A.cu ? kv_item_of(A.cu, A.n_items, token) : token;
        if (tid == 0) item_sh = i;
    }
    __syncthreads();
    const int item = item_sh;
    if (item >= A.n_items) return;
    const int first = A.cu ? A.cu[item] : token, count = A.cu ? A.cu[item + 1] - first : 1;
    const int seq = kv_sequence(A.c, A.seqs, item);
    const int length = seq < 0 ? 0 : kv_length(A.c, seq);
    const int pos = length - count + (token - first);
    int hi = min(A.causal ? pos + 1 : length, A.max_len);
    const int lo = A.window > 0 ? max(0, pos - A.window + 1) : 0;
    if (token - first >= A.max_tokens) hi = 0;
    const int ps = 1 << A.c.page_log;
    for (int g = 0; g < A.group; ++g) {
        const int h = head * A.group + g;
        __syncthreads();
        {
            const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(A.q) + token * A.q_token + h * A.q_head;
            q[tid] = tid < A.d ? __bfloat162float(x[tid]) : 0.f;
            for (int s = 1; s < 128; s <<= 1) {
                __syncthreads();
                const float a = q[tid], b = q[tid ^ s];
                __syncthreads();
                q[tid] = (tid & s) ? b - a : a + b;
            }
            __syncthreads();
        }
        float m = -INFINITY, l = 0.f, o = 0.f;
        for (int t0 = lo; t0 < hi; t0 += TILE) {
            const int t = t0 + tid;
            float s = -INFINITY;
            const unsigned char* block = nullptr;
            if (t < hi) {
                const int page = kv_page(A.c, seq, t);
                if (page >= 0) block = kv_block(A.c, page, head);
            }
            float vs = 0.f, vl = 0.f;
            if (block) {
                const int slot = t & (ps - 1);
                const unsigned char* codes = block + slot * KV_ROW;
                float dot = 0.f, sum = 0.f;
                for (int j = 0; j < 128; ++j) {
                    const int c = (codes[j >> 1] >> (4 * (j & 1))) & 15;
                    dot = fmaf(q[j], (float)(ASYM ? c : (c ^ 8) - 8), dot);
                    sum += q[j];
                }
                const float* sc = reinterpret_cast<const float*>(block + 2 * ps * KV_ROW);
                if (ASYM) {
                    s = dot * sc[2 * slot] + sum * sc[2 * slot + 1];
                    vs = sc[2 * (ps + slot)];
                    vl = sc[2 * (ps + slot) + 1];
                } else {
                    s = dot * sc[slot];
                    vs = sc[ps + slot];
                }
                s *= A.scale * KV_NORM;
            }
            float mx = s;
            for (int k = 16; k; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
            __syncthreads();
            if ((tid & 31) == 0) red[tid >> 5] = mx;
            __syncthreads();
            mx = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
            const float e = block ? expf(s - mx) : 0.f;
            const float keep = mx > -INFINITY ? expf(m - mx) : 1.f;
            p[tid] = block ? e * vs : 0.f;
            add[tid] = block ? e * vl : 0.f;
            float sum = e;
            for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
            __syncthreads();
            if ((tid & 31) == 0) red[tid >> 5] = sum;
            __syncthreads();
            l = l * keep + red[0] + red[1] + red[2] + red[3];
            o *= keep;
            m = mx;
            for (int j = 0; j < min(TILE, hi - t0); ++j) {
                const int page = kv_page(A.c, seq, t0 + j);
                if (page < 0) continue;
                const unsigned char* codes = kv_block(A.c, page, head) + ps * KV_ROW + ((t0 + j) & (ps - 1)) * KV_ROW;
                const int c = (codes[tid >> 1] >> (4 * (tid & 1))) & 15;
                o = fmaf(p[j], (float)(ASYM ? c : (c ^ 8) - 8), o) + add[j];
            }
        }
        __syncthreads();
        q[tid] = l > 0.f || l != l ? o / l * KV_NORM : 0.f;
        for (int s = 1; s < 128; s <<= 1) {
            __syncthreads();
            const float a = q[tid], b = q[tid ^ s];
            __syncthreads();
            q[tid] = (tid & s) ? b - a : a + b;
        }
        if (tid < A.d) (static_cast<__nv_bfloat16*>(A.out) + token * A.out_token + h * A.out_head)[tid] = __float2bfloat16(q[tid]);
    }
}

}  // namespace

int64_t gbs_kv_attn_workspace(const gbs_plan*, int, int) { return 16; }

int gbs_kv_attn_launch(const gbs_plan* p, const gbs_kv_attn& A, void*, cudaStream_t stream)
{
    return gbs_kv_launch(p, p->asym ? k_kv_attn_plain<true> : k_kv_attn_plain<false>, dim3((unsigned)A.n_tokens, (unsigned)A.c.heads), THREADS, 0,
                         stream, A);
}
