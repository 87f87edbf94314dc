// C-ABI entry points of the paged KV cache: argument checks and dispatch.  Every error that the host can see is caught here, before
// anything is launched; what only the device knows (lengths, page numbers) the kernels check.
#include <math.h>

#include <algorithm>

#include "gbs_internal.h"

namespace {

bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_plan(const gbs_plan* p)
{
    if (!p) return GBS_ERR_INVALID_ARG;
    return p->bits == 4 && p->d_pad == 128 && p->m == 1 && (p->group == 0 || p->group == 128) && p->d % 8 == 0 ? GBS_OK : GBS_ERR_UNSUPPORTED;
}

int log2_page(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : page_size == 128 ? 7 : -1; }

int view_of(const gbs_plan* p, const gbs_kv_cache_t* c, gbs_kv_view* out)
{
    const int rc = check_plan(p);
    if (rc != GBS_OK) return rc;
    if (!c) return GBS_ERR_INVALID_ARG;
    const int page_log = log2_page(c->page_size);
    if (page_log < 0 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return GBS_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->n_pages > 1ll << 30 || c->n_seqs < 1 || c->max_pages < 1) return GBS_ERR_INVALID_ARG;
    if (c->max_pages > 1 << 20) return GBS_ERR_INVALID_ARG;          // positions fit 27 bits, and the pages that 1024 items want 30
    if (!c->pages || !c->page_table || !c->lengths || !c->refs) return GBS_ERR_INVALID_ARG;
    if (!aligned(c->pages, 16) || !aligned(c->page_table, 4) || !aligned(c->lengths, 4) || !aligned(c->refs, 4)) return GBS_ERR_ALIGNMENT;
    out->pages = static_cast<unsigned char*>(c->pages);
    out->page_table = c->page_table;
    out->lengths = c->lengths;
    out->refs = c->refs;
    out->n_pages = (int)c->n_pages;
    out->heads = c->n_kv_heads;
    out->page_log = page_log;
    out->n_seqs = c->n_seqs;
    out->max_pages = c->max_pages;
    out->block_bytes = c->page_size * (128 + 8 * (p->asym ? 2 : 1));
    out->page_bytes = (long long)out->block_bytes * c->n_kv_heads;
    return GBS_OK;
}

int check_items(const gbs_kv_view& v, const int32_t* seqs, int n_items)
{
    if (n_items < 0 || n_items > GBS_KV_MAX_ITEMS) return GBS_ERR_INVALID_ARG;
    if (!seqs && n_items > v.n_seqs) return GBS_ERR_INVALID_ARG;
    return aligned(seqs, 4) ? GBS_OK : GBS_ERR_ALIGNMENT;
}

// items and the rows of a call; *empty: nothing to do
int check_tokens(const gbs_kv_view& v, const int32_t* seqs, const int32_t* cu, int n_items, int64_t n_tokens, bool* empty)
{
    const int rc = check_items(v, seqs, n_items);
    if (rc != GBS_OK) return rc;
    if (n_tokens < 0 || n_tokens >= 1ll << 30 || n_tokens * v.heads >= 1ll << 30 || (!cu && n_tokens != n_items)) return GBS_ERR_INVALID_ARG;
    *empty = n_items == 0 || n_tokens == 0;
    return aligned(cu, 4) ? GBS_OK : GBS_ERR_ALIGNMENT;
}

int check_strides(const gbs_plan* p, int64_t token, int64_t head)
{
    if (token < p->d || head < p->d) return GBS_ERR_INVALID_ARG;
    return (token | head) & 7 ? GBS_ERR_ALIGNMENT : GBS_OK;
}

// the launch, on the plan's device; a failed one is reported once, here
template <typename F>
int on_device(const gbs_plan* p, F launch)
{
    gbs_device_guard g;
    if (g.enter(p->device) != cudaSuccess) {
        cudaGetLastError();
        return GBS_ERR_CUDA;
    }
    const int e = launch();
    if (e != 0) cudaGetLastError();
    return e == 0 ? GBS_OK : GBS_ERR_CUDA;
}

}  // namespace

extern "C" int gbs_kv_page_bytes(const gbs_plan_t* p, int n_kv_heads, int page_size, int64_t* out)
{
    const int rc = check_plan(p);
    if (rc != GBS_OK) return rc;
    if (!out || n_kv_heads < 1 || n_kv_heads > 1024 || log2_page(page_size) < 0) return GBS_ERR_INVALID_ARG;
    *out = (int64_t)n_kv_heads * page_size * (128 + 8 * (p->asym ? 2 : 1));
    return GBS_OK;
}

extern "C" int gbs_kv_extend(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* counts, int n_items,
                             int32_t* status_out, void* stream)
{
    gbs_kv_view v;
    int rc = view_of(p, cache, &v);
    if (rc == GBS_OK) rc = check_items(v, seqs, n_items);
    if (rc != GBS_OK || n_items == 0) return rc;
    if (!status_out) return GBS_ERR_INVALID_ARG;
    if (!aligned(counts, 4) || !aligned(status_out, 4)) return GBS_ERR_ALIGNMENT;
    return on_device(p, [&] { return gbs_kv_extend_launch(p, v, seqs, counts, n_items, status_out, static_cast<cudaStream_t>(stream)); });
}

extern "C" int gbs_kv_fork(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* src, const int32_t* dst, int n_items,
                           int32_t* status_out, void* stream)
{
    gbs_kv_view v;
    int rc = view_of(p, cache, &v);
    if (rc != GBS_OK) return rc;
    if (n_items < 0 || n_items > GBS_KV_MAX_ITEMS) return GBS_ERR_INVALID_ARG;
    if (n_items == 0) return GBS_OK;
    if (!src || !dst || !status_out) return GBS_ERR_INVALID_ARG;
    if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(status_out, 4)) return GBS_ERR_ALIGNMENT;
    return on_device(p, [&] { return gbs_kv_fork_launch(p, v, src, dst, n_items, status_out, static_cast<cudaStream_t>(stream)); });
}

extern "C" int gbs_kv_free(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, int n_items, void* stream)
{
    gbs_kv_view v;
    int rc = view_of(p, cache, &v);
    if (rc == GBS_OK) rc = check_items(v, seqs, n_items);
    if (rc != GBS_OK || n_items == 0) return rc;
    return on_device(p, [&] { return gbs_kv_free_launch(p, v, seqs, n_items, static_cast<cudaStream_t>(stream)); });
}

extern "C" int gbs_kv_compact(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const gbs_kv_cache_t* into, int32_t* page_map, int32_t* n_live,
                              void* stream)
{
    gbs_kv_view v, w;
    int rc = view_of(p, cache, &v);
    if (rc == GBS_OK) rc = view_of(p, into, &w);
    if (rc != GBS_OK) return rc;
    if (v.heads != w.heads || v.page_log != w.page_log || v.n_seqs != w.n_seqs || v.max_pages != w.max_pages) return GBS_ERR_INVALID_ARG;
    if (v.pages == w.pages || v.page_table == w.page_table || v.lengths == w.lengths || v.refs == w.refs) return GBS_ERR_INVALID_ARG;
    if (!page_map || !n_live) return GBS_ERR_INVALID_ARG;
    if (!aligned(page_map, 4) || !aligned(n_live, 4)) return GBS_ERR_ALIGNMENT;
    return on_device(p, [&] { return gbs_kv_compact_launch(p, v, w, page_map, n_live, static_cast<cudaStream_t>(stream)); });
}

extern "C" int gbs_kv_append_extended(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens,
                                      int n_items, int64_t n_tokens, const void* k, const void* v, int64_t token_stride, int64_t head_stride,
                                      const int32_t* status, void* stream)
{
    gbs_kv_view c;
    bool empty = false;
    int rc = view_of(p, cache, &c);
    if (rc == GBS_OK) rc = check_tokens(c, seqs, cu_tokens, n_items, n_tokens, &empty);
    if (rc != GBS_OK || empty) return rc;
    if (!k || !v) return GBS_ERR_INVALID_ARG;
    rc = check_strides(p, token_stride, head_stride);
    if (rc != GBS_OK) return rc;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(status, 4)) return GBS_ERR_ALIGNMENT;
    return on_device(p, [&] {
        return gbs_kv_append_launch(p, c, seqs, cu_tokens, n_items, n_tokens, k, v, token_stride, head_stride, status, static_cast<cudaStream_t>(stream));
    });
}

extern "C" int gbs_kv_append(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                             int64_t n_tokens, const void* k, const void* v, int64_t token_stride, int64_t head_stride, void* stream)
{
    return gbs_kv_append_extended(p, cache, seqs, cu_tokens, n_items, n_tokens, k, v, token_stride, head_stride, nullptr, stream);
}

extern "C" int gbs_kv_read(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                           int64_t n_tokens, void* k_out, void* v_out, void* stream)
{
    gbs_kv_view c;
    bool empty = false;
    int rc = view_of(p, cache, &c);
    if (rc == GBS_OK) rc = check_tokens(c, seqs, cu_tokens, n_items, n_tokens, &empty);
    if (rc != GBS_OK || empty) return rc;
    if (!k_out || !v_out) return GBS_ERR_INVALID_ARG;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return GBS_ERR_ALIGNMENT;
    return on_device(p, [&] { return gbs_kv_read_launch(p, c, seqs, cu_tokens, n_items, n_tokens, k_out, v_out, static_cast<cudaStream_t>(stream)); });
}

namespace {

// tiles of 8 rows up to here, of 256 beyond
bool few_rows(int group, int max_tokens) { return (int64_t)max_tokens * group <= GBS_KV_FEW_ROWS; }

int64_t workspace_bytes_of(const gbs_plan* p, int group, int max_tokens)
{
    return few_rows(group, max_tokens) ? gbs_kv_few_workspace(p) : gbs_tc_kvattn_workspace(p);
}

int check_heads(const gbs_kv_view& c, int n_heads, int max_tokens, bool ragged)
{
    if (n_heads < 1 || n_heads % c.heads != 0 || n_heads / c.heads > 1024) return GBS_ERR_INVALID_ARG;
    if (max_tokens < 1 || (!ragged && max_tokens != 1)) return GBS_ERR_INVALID_ARG;
    return (int64_t)max_tokens * (n_heads / c.heads) <= 1ll << 28 ? GBS_OK : GBS_ERR_INVALID_ARG;
}

}  // namespace

extern "C" int gbs_kv_attention_workspace(const gbs_plan_t* p, const gbs_kv_cache_t* cache, int n_heads, int64_t n_tokens, int max_tokens,
                                          int64_t* bytes_out)
{
    gbs_kv_view c;
    int rc = view_of(p, cache, &c);
    if (rc == GBS_OK) rc = check_heads(c, n_heads, max_tokens, true);
    if (rc != GBS_OK) return rc;
    if (!bytes_out || n_tokens < 0) return GBS_ERR_INVALID_ARG;
    *bytes_out = workspace_bytes_of(p, n_heads / c.heads, max_tokens);
    return GBS_OK;
}

namespace {

struct AttnCall {
    const int32_t *seqs, *cu_tokens;
    int n_items;
    int64_t n_tokens;
    int max_tokens, max_len;
    const void* q;
    int64_t q_token, q_head;
    int n_heads;
    float scale;
    int window, flags;
    void* out;
    int64_t out_token, out_head;
};

// What the calls that attend check alike, and the kernels' arguments; *empty: nothing to do.  A call without `out` has other results.
int attn_args(const gbs_plan* p, const gbs_kv_cache_t* cache, const AttnCall& x, gbs_kv_attn* to, bool* empty)
{
    gbs_kv_attn A = {};
    int rc = view_of(p, cache, &A.c);
    if (rc == GBS_OK) rc = check_tokens(A.c, x.seqs, x.cu_tokens, x.n_items, x.n_tokens, empty);
    if (rc == GBS_OK) rc = check_heads(A.c, x.n_heads, x.max_tokens, x.cu_tokens != nullptr);
    if (rc != GBS_OK) return rc;
    if ((x.flags & ~GBS_KV_CAUSAL) || x.window < 0 || x.max_len < 0 || !isfinite(x.scale)) return GBS_ERR_INVALID_ARG;
    if (x.n_tokens * x.n_heads >= 1ll << 31 || (int64_t)x.n_items * x.max_tokens * (x.n_heads / A.c.heads) > 1ll << 28) return GBS_ERR_INVALID_ARG;
    A.seqs = x.seqs;
    A.cu = x.cu_tokens;
    A.n_items = x.n_items;
    A.max_tokens = (int)std::min<int64_t>(x.max_tokens, x.n_tokens);
    A.max_len = x.max_len > 0 ? x.max_len : A.c.max_pages << A.c.page_log;
    A.window = std::min(x.window, 1 << 30);                          // beyond any position: position - window stays within 32 bits
    A.causal = x.flags & GBS_KV_CAUSAL;
    A.n_heads = x.n_heads;
    A.group = x.n_heads / A.c.heads;
    A.by_group.set((unsigned)A.group);
    A.d = p->d;
    A.scale = x.scale == 0.f ? (float)(1.0 / sqrt((double)p->d)) : x.scale;
    A.n_tokens = x.n_tokens;
    A.q = x.q;
    A.out = x.out;
    A.q_token = x.q_token;
    A.q_head = x.q_head;
    A.out_token = x.out_token;
    A.out_head = x.out_head;
    *to = A;
    return GBS_OK;
}
// the call's tensors
int check_rows(const gbs_plan* p, const AttnCall& x, bool has_out, const void* workspace)
{
    int rc = check_strides(p, x.q_token, x.q_head);
    if (rc == GBS_OK && has_out) rc = check_strides(p, x.out_token, x.out_head);
    if (rc != GBS_OK) return rc;
    if (!aligned(x.q, 16) || !aligned(x.out, 16) || !aligned(workspace, 16)) return GBS_ERR_ALIGNMENT;
    return x.q == x.out ? GBS_ERR_INVALID_ARG : GBS_OK;              // rows are read after others have been written
}

// waits of the attention kernels, for few rows and for many
bool selftest_code(int code) { return (code >= 61 && code <= 64) || (code >= 71 && code <= 77); }

// code, segment: of the waits that count as run out in the self-test (0: none)
int attention(const gbs_plan* p, const gbs_kv_cache_t* cache, const AttnCall& x, void* workspace, int64_t workspace_bytes, int code, int segment, void* stream)
{
    gbs_kv_attn A;
    bool empty = false;
    int rc = attn_args(p, cache, x, &A, &empty);
    if (rc != GBS_OK || empty) return rc;
    if (!x.q || !x.out || !workspace || workspace_bytes < workspace_bytes_of(p, A.group, x.max_tokens)) return GBS_ERR_INVALID_ARG;
    rc = check_rows(p, x, true, workspace);
    if (rc != GBS_OK) return rc;
    A.lost_code = code;
    A.lost_segment = segment;
    return on_device(p, [&] {
        return few_rows(A.group, x.max_tokens) ? gbs_kv_few_launch(p, A, workspace, static_cast<cudaStream_t>(stream))
                                               : gbs_tc_kvattn_launch(p, A, workspace, static_cast<cudaStream_t>(stream));
    });
}

}  // namespace

extern "C" int gbs_kv_attention(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                int64_t n_tokens, int max_tokens, int max_len, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                                int n_heads, float scale, int window, int flags, void* out, int64_t out_token_stride,
                                int64_t out_head_stride, void* workspace, int64_t workspace_bytes, void* stream)
{
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, max_len, q, q_token_stride, q_head_stride, n_heads,
                        scale, window, flags, out, out_token_stride, out_head_stride};
    return attention(p, cache, x, workspace, workspace_bytes, 0, 0, stream);
}

extern "C" int gbs_selftest_kv_attention(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                         int64_t n_tokens, int max_tokens, int max_len, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                                         int n_heads, float scale, int window, int flags, void* out, int64_t out_token_stride,
                                         int64_t out_head_stride, void* workspace, int64_t workspace_bytes, int code, int segment, void* stream)
{
    if (!selftest_code(code) || segment < 0) return GBS_ERR_INVALID_ARG;
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, max_len, q, q_token_stride, q_head_stride, n_heads,
                        scale, window, flags, out, out_token_stride, out_head_stride};
    return attention(p, cache, x, workspace, workspace_bytes, code, segment, stream);
}

namespace {

int check_groups(const int32_t* groups, int n_groups, const gbs_kv_attn& A)
{
    if (n_groups < 1 || n_groups > GBS_KV_MAX_ITEMS || (!groups && n_groups != 1)) return GBS_ERR_INVALID_ARG;
    if (A.n_tokens * A.group > 1ll << 28) return GBS_ERR_INVALID_ARG;
    return aligned(groups, 4) ? GBS_OK : GBS_ERR_ALIGNMENT;
}

// the sizes that a workspace goes by
int sizes_of(const gbs_plan* p, const gbs_kv_cache_t* cache, int n_items, int64_t n_tokens, int max_tokens, int n_heads, const int64_t* bytes_out,
             gbs_kv_attn* to)
{
    gbs_kv_attn A = {};
    int rc = view_of(p, cache, &A.c);
    if (rc == GBS_OK) rc = check_heads(A.c, n_heads, max_tokens, true);
    if (rc != GBS_OK) return rc;
    if (!bytes_out || n_items < 0 || n_items > GBS_KV_MAX_ITEMS) return GBS_ERR_INVALID_ARG;
    if (n_tokens < 0 || n_tokens >= 1ll << 30 || n_tokens * n_heads >= 1ll << 31 || n_tokens * (n_heads / A.c.heads) > 1ll << 28) return GBS_ERR_INVALID_ARG;
    A.n_items = n_items;
    A.n_tokens = n_tokens;
    A.max_tokens = (int)std::min<int64_t>(max_tokens, n_tokens);     // as in the call
    A.n_heads = n_heads;
    A.group = n_heads / A.c.heads;
    *to = A;
    return GBS_OK;
}

}  // namespace

extern "C" int gbs_kv_shared_attention_workspace(const gbs_plan_t* p, const gbs_kv_cache_t* cache, int n_items, int64_t n_tokens, int max_tokens,
                                                 int n_groups, int max_prefix, int n_heads, int64_t* bytes_out)
{
    gbs_kv_attn A;
    const int rc = sizes_of(p, cache, n_items, n_tokens, max_tokens, n_heads, bytes_out, &A);
    if (rc != GBS_OK) return rc;
    if (n_groups < 1 || n_groups > GBS_KV_MAX_ITEMS || max_prefix < 0) return GBS_ERR_INVALID_ARG;
    *bytes_out = gbs_kv_shared_workspace(p, A, n_groups, max_prefix);
    return GBS_OK;
}

namespace {

// code, segment: as for attention
int shared_attention(const gbs_plan* p, const gbs_kv_cache_t* cache, const AttnCall& x, const int32_t* groups, int n_groups, int max_prefix, void* workspace,
                     int64_t workspace_bytes, int code, int segment, void* stream)
{
    gbs_kv_attn A;
    bool empty = false;
    int rc = attn_args(p, cache, x, &A, &empty);
    if (rc == GBS_OK) rc = max_prefix < 0 ? GBS_ERR_INVALID_ARG : check_groups(groups, n_groups, A);
    if (rc != GBS_OK || empty) return rc;
    if (!x.q || !x.out || !workspace || workspace_bytes < gbs_kv_shared_workspace(p, A, n_groups, max_prefix)) return GBS_ERR_INVALID_ARG;
    rc = check_rows(p, x, true, workspace);
    if (rc != GBS_OK) return rc;
    A.lost_code = code;
    A.lost_segment = segment;
    return on_device(p, [&] { return gbs_kv_shared_launch(p, A, groups, n_groups, max_prefix, workspace, static_cast<cudaStream_t>(stream)); });
}

}  // namespace

extern "C" int gbs_kv_shared_attention(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                       int64_t n_tokens, int max_tokens, const int32_t* groups, int n_groups, int max_own, int max_prefix, const void* q,
                                       int64_t q_token_stride, int64_t q_head_stride, int n_heads, float scale, int flags, void* out,
                                       int64_t out_token_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes, void* stream)
{
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, max_own, q, q_token_stride, q_head_stride, n_heads,
                        scale, 0, flags, out, out_token_stride, out_head_stride};
    return shared_attention(p, cache, x, groups, n_groups, max_prefix, workspace, workspace_bytes, 0, 0, stream);
}

extern "C" int gbs_selftest_kv_shared_attention(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                                int64_t n_tokens, int max_tokens, const int32_t* groups, int n_groups, int max_own, int max_prefix, const void* q,
                                                int64_t q_token_stride, int64_t q_head_stride, int n_heads, float scale, int flags, void* out,
                                                int64_t out_token_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes, int code,
                                                int segment, void* stream)
{
    if (!selftest_code(code) || segment < 0) return GBS_ERR_INVALID_ARG;
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, max_own, q, q_token_stride, q_head_stride, n_heads,
                        scale, 0, flags, out, out_token_stride, out_head_stride};
    return shared_attention(p, cache, x, groups, n_groups, max_prefix, workspace, workspace_bytes, code, segment, stream);
}

extern "C" int gbs_kv_attention_mass_workspace(const gbs_plan_t* p, const gbs_kv_cache_t* cache, int n_items, int64_t n_tokens, int max_tokens,
                                               int n_heads, int64_t width, int64_t* bytes_out)
{
    gbs_kv_attn A;
    const int rc = sizes_of(p, cache, n_items, n_tokens, max_tokens, n_heads, bytes_out, &A);
    if (rc != GBS_OK) return rc;
    if (width < 1) return GBS_ERR_INVALID_ARG;
    *bytes_out = gbs_kv_mass_workspace(p, A, width);
    return GBS_OK;
}

namespace {

// code, segment: as for attention
int attention_mass(const gbs_plan* p, const gbs_kv_cache_t* cache, const AttnCall& x, const float* base, float decay, float* mass, int64_t width,
                   void* workspace, int64_t workspace_bytes, int code, int segment, void* stream)
{
    gbs_kv_attn A;
    bool empty = false;
    int rc = attn_args(p, cache, x, &A, &empty);
    if (rc != GBS_OK) return rc;
    if (width < 1 || !isfinite(decay) || A.n_tokens * A.group > 1ll << 28) return GBS_ERR_INVALID_ARG;
    if (empty) return GBS_OK;
    if (!x.q || !mass || (!base && decay != 0.f) || !workspace || workspace_bytes < gbs_kv_mass_workspace(p, A, width)) return GBS_ERR_INVALID_ARG;
    rc = check_rows(p, x, false, workspace);
    if (rc != GBS_OK) return rc;
    if (!aligned(mass, 4) || !aligned(base, 4)) return GBS_ERR_ALIGNMENT;
    A.lost_code = code;
    A.lost_segment = segment;
    return on_device(p, [&] { return gbs_kv_mass_launch(p, A, base, decay, mass, width, workspace, static_cast<cudaStream_t>(stream)); });
}

}  // namespace

extern "C" int gbs_kv_attention_mass(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                     int64_t n_tokens, int max_tokens, const void* q, int64_t q_token_stride, int64_t q_head_stride, int n_heads,
                                     float scale, int window, int flags, const float* base, float decay, float* mass, int64_t width,
                                     void* workspace, int64_t workspace_bytes, void* stream)
{
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, 0, q, q_token_stride, q_head_stride, n_heads, scale, window, flags, nullptr, 0, 0};
    return attention_mass(p, cache, x, base, decay, mass, width, workspace, workspace_bytes, 0, 0, stream);
}

extern "C" int gbs_selftest_kv_attention_mass(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, const int32_t* cu_tokens, int n_items,
                                              int64_t n_tokens, int max_tokens, const void* q, int64_t q_token_stride, int64_t q_head_stride, int n_heads,
                                              float scale, int window, int flags, const float* base, float decay, float* mass, int64_t width,
                                              void* workspace, int64_t workspace_bytes, int code, int segment, void* stream)
{
    if (!((code >= 81 && code <= 86) || (code >= 91 && code <= 99)) || segment < 0) return GBS_ERR_INVALID_ARG;
    const AttnCall x = {seqs, cu_tokens, n_items, n_tokens, max_tokens, 0, q, q_token_stride, q_head_stride, n_heads, scale, window, flags, nullptr, 0, 0};
    return attention_mass(p, cache, x, base, decay, mass, width, workspace, workspace_bytes, code, segment, stream);
}

namespace {

// pages of the tokens that a sequence keeps, and the workspace: their numbers, a count of each item, and the weights of what stays
int keep_pages_of(const gbs_kv_view& c, int keep) { return std::min((int)(((int64_t)keep + (1 << c.page_log) - 1) >> c.page_log), c.max_pages); }
int64_t evict_numbers(const gbs_kv_view& c, int n_items, int keep) { return (int64_t)n_items * (keep_pages_of(c, keep) + 1); }
int64_t evict_bytes(const gbs_kv_view& c, int n_items, int keep)
{
    // no more tokens stay than a sequence can have
    const int64_t most = std::min<int64_t>(keep, (int64_t)c.max_pages << c.page_log);
    return (evict_numbers(c, n_items, keep) + n_items * c.heads * most) * 4;
}

}  // namespace

extern "C" int gbs_kv_evict_workspace(const gbs_plan_t* p, const gbs_kv_cache_t* cache, int n_items, int keep, int64_t* bytes_out)
{
    gbs_kv_view c;
    const int rc = view_of(p, cache, &c);
    if (rc != GBS_OK) return rc;
    if (!bytes_out || n_items < 0 || n_items > GBS_KV_MAX_ITEMS || keep < 1) return GBS_ERR_INVALID_ARG;
    *bytes_out = evict_bytes(c, n_items, keep);
    return GBS_OK;
}

extern "C" int gbs_kv_evict(const gbs_plan_t* p, const gbs_kv_cache_t* cache, const int32_t* seqs, int n_items, int keep, int recent, int first,
                            const float* mass, float* mass_out, int64_t width, int32_t* kept, int32_t* status_out, void* workspace,
                            int64_t workspace_bytes, void* stream)
{
    gbs_kv_eviction E = {};
    int rc = view_of(p, cache, &E.c);
    if (rc == GBS_OK) rc = check_items(E.c, seqs, n_items);
    if (rc != GBS_OK) return rc;
    if (keep < 1 || recent < 0 || first < 0 || (int64_t)recent + first > keep || width < 1) return GBS_ERR_INVALID_ARG;
    if (n_items == 0) return GBS_OK;
    E.keep_pages = keep_pages_of(E.c, keep);
    if (!mass || !mass_out || !kept || !status_out || !workspace || workspace_bytes < evict_bytes(E.c, n_items, keep)) return GBS_ERR_INVALID_ARG;
    if (!aligned(mass, 4) || !aligned(mass_out, 4) || !aligned(kept, 4) || !aligned(status_out, 4) || !aligned(workspace, 16)) return GBS_ERR_ALIGNMENT;
    E.seqs = seqs;
    E.n_items = n_items;
    E.keep = keep;
    E.recent = recent;
    E.first = first;
    E.mass = mass;
    E.mass_out = mass_out;
    E.width = width;
    E.status = status_out;
    E.kept = kept;
    E.fresh = static_cast<int*>(workspace);
    E.arrived = E.fresh + (int64_t)n_items * E.keep_pages;
    E.weights = reinterpret_cast<float*>(E.fresh) + evict_numbers(E.c, n_items, keep);
    return on_device(p, [&] { return gbs_kv_evict_launch(p, E, static_cast<cudaStream_t>(stream)); });
}
