// Native call path of the Python binding: what Plan's methods do per call -- check the tensors, allocate the outputs,
// look up the current stream, call the C ABI -- in one C function each.
//
// A call on a few rows is bound by the host: the kernel takes 3 us, and the same steps in Python took 17.5 us per call
// (two torch.empty at 2.3 us, torch.cuda.current_stream at 3.3 us, argument checks, ctypes marshalling at 0.8 us and the
// launch itself at 2 us).
//
// Every function here handles the regular call only and answers None for anything else (a tensor of another type or
// device, a shape or stride that needs a view, an output that is too small, a non-zero status): that call then takes
// the Python path, which raises the error or makes the view.  Nothing is enqueued before the checks have passed.
//
// Two ways in: the module's functions, for a caller that has the plan's handle alone, and method objects that stand in the class
// under the names of Plan's methods, over the Python functions they were.  A method object binds like a function, so that a
// bound method keeps its plan, a subclass may override it and a class attribute may be replaced; it finds the plan's handle in the
// Calls object of the instance.  It saves the Python frame around each call (0.9 of 5.3 us for 16 rows); what it does not handle it
// passes to the function it wraps.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <stddef.h>
#include <string.h>

#include <algorithm>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "gbs.h"

namespace {

// -1: not a type the library takes
int dtype_code(at::ScalarType t)
{
    return t == at::kFloat ? GBS_DTYPE_F32 : (t == at::kBFloat16 ? GBS_DTYPE_BF16 : -1);
}

struct PlanRef {
    const gbs_plan_t* plan;
    gbs_plan_info_t info;
};

bool plan_of(PyObject* o, const gbs_plan_t** plan, gbs_plan_info_t* info)
{
    if (!PyLong_Check(o)) return false;
    *plan = static_cast<const gbs_plan_t*>(PyLong_AsVoidPtr(o));
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return gbs_plan_info(*plan, info) == GBS_OK;
}

// None: the current stream of the current device; else a stream object with a `cuda_stream` handle
bool stream_of(PyObject* o, void** stream)
{
    if (o == Py_None) {
        *stream = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (h) {
        *stream = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
    }
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

const at::Tensor* cuda_tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

// rows [.., d]: two-dimensional with contiguous rows, or contiguous of any other rank
bool rows_of(const at::Tensor* t, int d, int64_t* n_rows, int64_t* stride)
{
    const int64_t r = t->dim();
    if (r < 1 || t->size(r - 1) != d || t->stride(r - 1) != 1) return false;
    if (r == 2) {
        *n_rows = t->size(0);
        *stride = *n_rows > 1 ? t->stride(0) : (t->stride(0) > d ? t->stride(0) : d);
        return true;
    }
    if (!t->is_contiguous()) return false;
    *n_rows = t->numel() / d;
    *stride = d;
    return true;
}

bool buffer_ok(const at::Tensor* t, const at::Device& device, int64_t min_numel)
{
    return t && t->device() == device && t->is_contiguous() && t->numel() >= min_numel;
}

at::Tensor empty2(int64_t r, int64_t c, at::ScalarType dtype, const at::Device& device)
{
    return at::detail::empty_cuda({r, c}, dtype, device, std::nullopt);
}

// A C++ exception (an allocation that fails, a tensor without memory of its own) makes the call an irregular one.  Whatever can throw
// stands before the GIL is released: a tensor's pointer, in particular, is asked for before.
#define GBS_BEGIN try {
#define GBS_END } catch (...) { PyErr_Clear(); } Py_RETURN_NONE;

// rotate_quantize(plan, x, want_y, out, stream) -> (codes, scales, y) or None
// (a[0] is not looked at: the plan comes as `ref`)
PyObject* do_rotate_quantize(const PlanRef& ref, PyObject* const* a)
{
    GBS_BEGIN
    const gbs_plan_t* plan = ref.plan;
    const gbs_plan_info_t& info = ref.info;
    void* stream;
    int64_t rows, stride;
    const at::Tensor* x = cuda_tensor(a[1]);
    if (!x || !rows_of(x, info.d, &rows, &stride) || !stream_of(a[4], &stream)) Py_RETURN_NONE;
    const int dt = dtype_code(x->scalar_type());
    if (dt < 0) Py_RETURN_NONE;
    const at::Device device = x->device();
    if (a[3] != Py_None) {
        if (!PyTuple_Check(a[3]) || PyTuple_GET_SIZE(a[3]) != 3) Py_RETURN_NONE;
        PyObject *oc = PyTuple_GET_ITEM(a[3], 0), *os = PyTuple_GET_ITEM(a[3], 1), *oy = PyTuple_GET_ITEM(a[3], 2);
        const at::Tensor *codes = cuda_tensor(oc), *scales = cuda_tensor(os), *y = oy == Py_None ? nullptr : cuda_tensor(oy);
        if (!buffer_ok(codes, device, rows * info.code_bytes_per_row) || codes->scalar_type() != at::kByte ||
            !buffer_ok(scales, device, rows * info.scale_floats_per_row) || scales->scalar_type() != at::kFloat ||
            (oy != Py_None && (!buffer_ok(y, device, rows * info.d_pad) || y->scalar_type() != at::kFloat)))
            Py_RETURN_NONE;
        void *xp = x->data_ptr(), *cp = codes->data_ptr(), *sp = scales->data_ptr(), *yp = y ? y->data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = gbs_rotate_quantize(plan, xp, dt, rows, stride, cp, static_cast<float*>(sp), static_cast<float*>(yp), stream);
        Py_END_ALLOW_THREADS
        if (rc != GBS_OK) Py_RETURN_NONE;
        Py_INCREF(a[3]);
        return a[3];
    }
    const int want_y = PyObject_IsTrue(a[2]);
    if (want_y < 0) { PyErr_Clear(); Py_RETURN_NONE; }
    // two allocations (0.5 us each): outputs that shared one would be saved, kept and freed together
    at::Tensor codes = empty2(rows, info.code_bytes_per_row, at::kByte, device);
    at::Tensor scales = empty2(rows, info.scale_floats_per_row, at::kFloat, device), y;
    if (want_y) y = empty2(rows, info.d_pad, at::kFloat, device);
    void *xp = x->data_ptr(), *cp = codes.data_ptr(), *sp = scales.data_ptr(), *yp = want_y ? y.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = gbs_rotate_quantize(plan, xp, dt, rows, stride, cp, static_cast<float*>(sp), static_cast<float*>(yp), stream);
    Py_END_ALLOW_THREADS
    if (rc != GBS_OK) Py_RETURN_NONE;
    PyObject* out = PyTuple_New(3);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(codes)));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(scales)));
    if (want_y) PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(std::move(y)));
    else PyTuple_SET_ITEM(out, 2, Py_NewRef(Py_None));
    return out;
    GBS_END
}

// an output the caller passed, or a new one [r, c] of the dtype asked for; false: not the regular call
bool output_of(PyObject* o, PyObject* dtype, int64_t r, int64_t c, const at::Device& device, at::Tensor* out, int* dt)
{
    if (o != Py_None) {
        const at::Tensor* t = cuda_tensor(o);
        if (!buffer_ok(t, device, r * c)) return false;
        *out = *t;
    } else {
        if (dtype && !THPDtype_Check(dtype)) return false;
        const at::ScalarType st = dtype ? reinterpret_cast<THPDtype*>(dtype)->scalar_type : at::kFloat;      // null: not given
        if (dtype_code(st) < 0) return false;
        *out = empty2(r, c, st, device);
    }
    *dt = dtype_code(out->scalar_type());
    return *dt >= 0;
}

// dequantize(plan, codes, scales, inverse, dtype, out, stream) -> tensor or None
PyObject* do_dequantize(const PlanRef& ref, PyObject* const* a)
{
    GBS_BEGIN
    const gbs_plan_t* plan = ref.plan;
    const gbs_plan_info_t& info = ref.info;
    void* stream;
    const at::Tensor *codes = cuda_tensor(a[1]), *scales = cuda_tensor(a[2]);
    if (!codes || codes->dim() < 1) Py_RETURN_NONE;
    const int64_t rows = codes->size(0);
    const at::Device device = codes->device();
    const int inverse = PyObject_IsTrue(a[3]);
    if (inverse < 0) { PyErr_Clear(); Py_RETURN_NONE; }
    if (codes->scalar_type() != at::kByte || !buffer_ok(codes, device, rows * info.code_bytes_per_row) ||
        !buffer_ok(scales, device, rows * info.scale_floats_per_row) || scales->scalar_type() != at::kFloat ||
        !stream_of(a[6], &stream))
        Py_RETURN_NONE;
    at::Tensor out;
    int dt;
    if (!output_of(a[5], a[4], rows, inverse ? info.d : info.d_pad, device, &out, &dt)) Py_RETURN_NONE;
    void *cp = codes->data_ptr(), *sp = scales->data_ptr(), *op = out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = gbs_dequantize(plan, cp, static_cast<const float*>(sp), rows, op, dt, inverse ? GBS_INVERSE_ROTATE : 0, stream);
    Py_END_ALLOW_THREADS
    if (rc != GBS_OK) Py_RETURN_NONE;
    if (a[5] != Py_None) return Py_NewRef(a[5]);
    return THPVariable_Wrap(std::move(out));
    GBS_END
}

// quantized_matmul(plan_x, codes_x, scales_x, plan_w, codes_w, scales_w, dtype, out, stream) -> tensor or None
PyObject* do_quantized_matmul(const PlanRef& ref, PyObject* const* a)
{
    GBS_BEGIN
    const gbs_plan_t *px = ref.plan, *pw;
    const gbs_plan_info_t& ix = ref.info;
    gbs_plan_info_t iw;
    void* stream;
    if (!plan_of(a[3], &pw, &iw)) Py_RETURN_NONE;
    const at::Tensor *cx = cuda_tensor(a[1]), *sx = cuda_tensor(a[2]), *cw = cuda_tensor(a[4]), *sw = cuda_tensor(a[5]);
    if (!cx || !cw || cx->dim() < 1 || cw->dim() < 1) Py_RETURN_NONE;
    const int64_t n_tok = cx->size(0), n_out = cw->size(0);
    const at::Device device = cx->device();
    if (cx->scalar_type() != at::kByte || !buffer_ok(cx, device, n_tok * ix.code_bytes_per_row) ||
        !buffer_ok(sx, device, n_tok * ix.scale_floats_per_row) || sx->scalar_type() != at::kFloat ||
        cw->scalar_type() != at::kByte || !buffer_ok(cw, device, n_out * iw.code_bytes_per_row) ||
        !buffer_ok(sw, device, n_out * iw.scale_floats_per_row) || sw->scalar_type() != at::kFloat || !stream_of(a[8], &stream))
        Py_RETURN_NONE;
    at::Tensor out;
    int dt;
    // a caller's `out` may have any row stride: that form keeps the Python path's checks
    if (a[7] != Py_None) {
        const at::Tensor* t = cuda_tensor(a[7]);
        if (!t || t->dim() != 2 || t->size(0) != n_tok || t->size(1) != n_out) Py_RETURN_NONE;
    }
    if (!output_of(a[7], a[6], n_tok, n_out, device, &out, &dt)) Py_RETURN_NONE;
    void *cxp = cx->data_ptr(), *sxp = sx->data_ptr(), *cwp = cw->data_ptr(), *swp = sw->data_ptr(), *op = out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = gbs_quantized_matmul(px, cxp, static_cast<const float*>(sxp), n_tok, pw, cwp, static_cast<const float*>(swp), n_out, op, dt, n_out,
                              stream);
    Py_END_ALLOW_THREADS
    if (rc != GBS_OK) Py_RETURN_NONE;
    if (a[7] != Py_None) return Py_NewRef(a[7]);
    return THPVariable_Wrap(std::move(out));
    GBS_END
}

// clip_error(plan, x, alphas, stream) -> a new tensor of the K error sums, or None
PyObject* do_clip_error(const PlanRef& ref, PyObject* const* a)
{
    GBS_BEGIN
    const gbs_plan_t* plan = ref.plan;
    const gbs_plan_info_t& info = ref.info;
    void* stream;
    int64_t rows, stride;
    const at::Tensor* x = cuda_tensor(a[1]);
    if (!x || !rows_of(x, info.d, &rows, &stride) || !stream_of(a[3], &stream)) Py_RETURN_NONE;
    const int dt = dtype_code(x->scalar_type());
    if (dt < 0 || !PySequence_Check(a[2])) Py_RETURN_NONE;
    const Py_ssize_t K = PySequence_Size(a[2]);
    if (K < 1 || K > GBS_MAX_CANDIDATES) { PyErr_Clear(); Py_RETURN_NONE; }
    float alphas[GBS_MAX_CANDIDATES];
    for (Py_ssize_t i = 0; i < K; ++i) {
        PyObject* v = PySequence_GetItem(a[2], i);
        if (v) {
            alphas[i] = static_cast<float>(PyFloat_AsDouble(v));
            Py_DECREF(v);
        }
        if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
        if (!(alphas[i] > 0.f) || !(alphas[i] <= 1.f)) Py_RETURN_NONE;
    }
    // the sums are zeroed on the stream that adds to them
    at::Tensor err = at::detail::empty_cuda({static_cast<int64_t>(K)}, at::kDouble, x->device(), std::nullopt);
    void *xp = x->data_ptr(), *ep = err.data_ptr();
    int rc = GBS_ERR_CUDA;
    Py_BEGIN_ALLOW_THREADS
    if (cudaMemsetAsync(ep, 0, sizeof(double) * static_cast<size_t>(K), static_cast<cudaStream_t>(stream)) == cudaSuccess)
        rc = gbs_clip_error(plan, xp, dt, rows, stride, alphas, static_cast<int>(K), static_cast<double*>(ep), nullptr, stream);
    else
        cudaGetLastError();                               // the Python path reports it; later launches of others must not
    Py_END_ALLOW_THREADS
    if (rc != GBS_OK) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(err));
    GBS_END
}

// ---- the module's functions: the plan's handle first
template <PyObject* (*F)(const PlanRef&, PyObject* const*), int N>
PyObject* with_handle(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    PlanRef ref;
    if (n != N || !plan_of(a[0], &ref.plan, &ref.info)) Py_RETURN_NONE;
    return F(ref, a);
}

// ---- Calls(handle): the plan's handle and sizes for the methods below, until clear()
struct Calls {
    PyObject_HEAD
    PlanRef ref;              // ref.plan is null once the plan is closed
};
PyTypeObject* calls_type = nullptr;

int calls_init(PyObject* self, PyObject* args, PyObject*)
{
    Calls* c = reinterpret_cast<Calls*>(self);
    PyObject *handle, *unused;
    if (!PyArg_ParseTuple(args, "O|O", &handle, &unused)) return -1;
    if (!plan_of(handle, &c->ref.plan, &c->ref.info)) {
        c->ref.plan = nullptr;
        PyErr_SetString(PyExc_ValueError, "gbs: not a plan handle");
        return -1;
    }
    return 0;
}
void calls_dealloc(PyObject* self)
{
    PyTypeObject* type = Py_TYPE(self);
    type->tp_free(self);
    Py_DECREF(type);
}
PyObject* calls_clear(PyObject* self, PyObject*)
{
    reinterpret_cast<Calls*>(self)->ref.plan = nullptr;
    Py_RETURN_NONE;
}

// ---- Pool(calls, pages, page_table, lengths, refs, n_kv_heads, page_size): what the native methods know of a KVCache
struct Pool {
    PyObject_HEAD
    PyObject* calls;          // the plan's Calls: says when the plan is closed
    gbs_kv_cache_t cache;     // the KVCache keeps the tensors
    int device;
};
PyTypeObject* pool_type = nullptr;
PyObject* name_calls = nullptr;

int pool_init(PyObject* self, PyObject* args, PyObject*)
{
    Pool* p = reinterpret_cast<Pool*>(self);
    PyObject *calls, *o[4];
    int heads, page;
    if (!PyArg_ParseTuple(args, "OOOOOii", &calls, &o[0], &o[1], &o[2], &o[3], &heads, &page)) return -1;
    const at::Tensor* t[4];
    for (int i = 0; i < 4; ++i) t[i] = cuda_tensor(o[i]);
    if (Py_TYPE(calls) != calls_type || !t[0] || !t[1] || !t[2] || !t[3] || t[1]->dim() != 2) {
        PyErr_SetString(PyExc_ValueError, "gbs: not a plan's calls and a pool's tensors");
        return -1;
    }
    try {
        p->cache = {t[0]->data_ptr(), t[0]->size(0), heads, page, static_cast<int32_t*>(t[1]->data_ptr()), static_cast<int32_t*>(t[2]->data_ptr()),
                    static_cast<int32_t*>(t[3]->data_ptr()), static_cast<int>(t[1]->size(0)), static_cast<int>(t[1]->size(1))};
        p->device = t[0]->device().index();
    } catch (...) {
        PyErr_SetString(PyExc_ValueError, "gbs: a pool's tensor has no memory");
        return -1;
    }
    Py_XSETREF(p->calls, Py_NewRef(calls));
    return 0;
}
void pool_dealloc(PyObject* self)
{
    PyTypeObject* type = Py_TYPE(self);
    Py_CLEAR(reinterpret_cast<Pool*>(self)->calls);
    type->tp_free(self);
    Py_DECREF(type);
}

// the plan of a pool, null once it is closed
const PlanRef* plan_ref(const Pool& p)
{
    const Calls* c = reinterpret_cast<const Calls*>(p.calls);
    return c && c->ref.plan ? &c->ref : nullptr;
}

// a row of n int32 on the pool's device; null stays null
bool ints_of(const Pool& p, PyObject* o, int64_t n, const int32_t** out)
{
    *out = nullptr;
    if (!o || o == Py_None) return true;
    const at::Tensor* t = cuda_tensor(o);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != n || !t->is_contiguous() || t->device().index() != p.device) return false;
    *out = static_cast<const int32_t*>(t->data_ptr());
    return true;
}
int64_t length_of(PyObject* o)
{
    if (!o || !THPVariable_Check(o)) return -1;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.dim() == 1 ? t.size(0) : -1;
}

struct Rows {
    const at::Tensor* t;
    void* ptr;
    int64_t n, heads, token, head;
};
// [tokens, heads, d] in bf16 with contiguous rows
bool rows3_of(const Pool& p, PyObject* o, int d, Rows* r)
{
    const at::Tensor* t = cuda_tensor(o);
    if (!t || t->scalar_type() != at::kBFloat16 || t->dim() != 3 || t->size(2) != d || t->stride(2) != 1 || t->device().index() != p.device) return false;
    *r = {t, t->data_ptr(), t->size(0), t->size(1), t->size(0) > 1 ? t->stride(0) : d, t->size(1) > 1 ? t->stride(1) : d};
    return true;
}

struct Items {
    const int32_t *seqs, *cu;
    int64_t n;
};
bool items_of(const Pool& p, PyObject* seqs, PyObject* cu, int64_t tokens, Items* it)
{
    const bool has_seqs = seqs && seqs != Py_None, has_cu = cu && cu != Py_None;
    it->n = has_seqs ? length_of(seqs) : has_cu ? length_of(cu) - 1 : tokens;
    return it->n >= 0 && it->n <= GBS_KV_MAX_ITEMS && ints_of(p, seqs, it->n, &it->seqs) && ints_of(p, cu, it->n + 1, &it->cu);
}

bool none(PyObject* o) { return !o || o == Py_None; }

// an int argument; absent: `standard`
bool int_of(PyObject* o, int standard, int* out)
{
    *out = standard;
    if (!o) return true;
    const long v = PyLong_Check(o) ? PyLong_AsLong(o) : -1;
    if (!PyLong_Check(o) || PyErr_Occurred() || v < 0 || v > 0x7fffffff) { PyErr_Clear(); return false; }
    *out = static_cast<int>(v);
    return true;
}

void* stream_on(const Pool& p) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(p.device)).stream(); }
at::Device device_of(const Pool& p) { return at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(p.device)); }
at::Tensor ints(const Pool& p, int64_t n) { return at::detail::empty_cuda({n}, at::kInt, device_of(p), std::nullopt); }

// The regular calls on a pool: on the current stream of its device.
PyObject* do_kv_extend(const Pool& p, const PlanRef& ref, PyObject* const* g)        // seqs, counts, stream
{
    GBS_BEGIN
    if (!none(g[2])) Py_RETURN_NONE;
    const int64_t n = !none(g[0]) ? length_of(g[0]) : !none(g[1]) ? length_of(g[1]) : p.cache.n_seqs;
    const int32_t *seqs, *counts;
    if (n < 0 || n > GBS_KV_MAX_ITEMS || !ints_of(p, g[0], n, &seqs) || !ints_of(p, g[1], n, &counts)) Py_RETURN_NONE;
    at::Tensor status = ints(p, n);
    int32_t* sp = static_cast<int32_t*>(status.data_ptr());
    if (gbs_kv_extend(ref.plan, &p.cache, seqs, counts, static_cast<int>(n), sp, stream_on(p)) != GBS_OK) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(status));
    GBS_END
}
PyObject* do_kv_fork(const Pool& p, const PlanRef& ref, PyObject* const* g)          // src, dst, stream
{
    GBS_BEGIN
    const int64_t n = length_of(g[0]);
    const int32_t *src, *dst;
    if (!none(g[2]) || n < 0 || n > GBS_KV_MAX_ITEMS || none(g[1]) || !ints_of(p, g[0], n, &src) || !ints_of(p, g[1], n, &dst)) Py_RETURN_NONE;
    at::Tensor status = ints(p, n);
    int32_t* sp = static_cast<int32_t*>(status.data_ptr());
    if (gbs_kv_fork(ref.plan, &p.cache, src, dst, static_cast<int>(n), sp, stream_on(p)) != GBS_OK) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(status));
    GBS_END
}
// Calls that return None answer True: None says that the call was not made.
PyObject* do_kv_free(const Pool& p, const PlanRef& ref, PyObject* const* g)          // seqs, stream
{
    GBS_BEGIN
    const int64_t n = length_of(g[0]);
    const int32_t* seqs;
    if (!none(g[1]) || n < 0 || n > GBS_KV_MAX_ITEMS || !ints_of(p, g[0], n, &seqs)) Py_RETURN_NONE;
    if (gbs_kv_free(ref.plan, &p.cache, seqs, static_cast<int>(n), stream_on(p)) != GBS_OK) Py_RETURN_NONE;
    Py_RETURN_TRUE;
    GBS_END
}
PyObject* do_kv_append(const Pool& p, const PlanRef& ref, PyObject* const* g)        // k, v, seqs, cu_tokens, stream, status
{
    GBS_BEGIN
    Rows k, v;
    Items it;
    const int32_t* status;
    if (!none(g[4]) || !rows3_of(p, g[0], ref.info.d, &k) || !rows3_of(p, g[1], ref.info.d, &v)) Py_RETURN_NONE;
    if (k.n != v.n || k.token != v.token || k.head != v.head || k.heads != p.cache.n_kv_heads || v.heads != k.heads) Py_RETURN_NONE;
    if (!items_of(p, g[2], g[3], k.n, &it) || !ints_of(p, g[5], it.n, &status)) Py_RETURN_NONE;
    if (gbs_kv_append_extended(ref.plan, &p.cache, it.seqs, it.cu, static_cast<int>(it.n), k.n, k.ptr, v.ptr, k.token, k.head, status,
                               stream_on(p)) != GBS_OK)
        Py_RETURN_NONE;
    Py_RETURN_TRUE;
    GBS_END
}
PyObject* do_kv_read(const Pool& p, const PlanRef& ref, PyObject* const* g)          // seqs, cu_tokens, n_tokens, out, stream
{
    GBS_BEGIN
    int n;
    Items it;
    if (!none(g[3]) || !none(g[4]) || none(g[2]) || !int_of(g[2], 0, &n) || !items_of(p, g[0], g[1], n, &it)) Py_RETURN_NONE;
    at::Tensor out[2];
    void* ptr[2];
    for (int i = 0; i < 2; ++i) {
        out[i] = at::detail::empty_cuda({n, p.cache.n_kv_heads, ref.info.d}, at::kBFloat16, device_of(p), std::nullopt);
        ptr[i] = out[i].data_ptr();
    }
    if (gbs_kv_read(ref.plan, &p.cache, it.seqs, it.cu, static_cast<int>(it.n), n, ptr[0], ptr[1], stream_on(p)) != GBS_OK) Py_RETURN_NONE;
    PyObject* t = PyTuple_New(2);
    if (!t) return nullptr;
    for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(t, i, THPVariable_Wrap(std::move(out[i])));
    return t;
    GBS_END
}
// q, seqs, cu_tokens, max_tokens, causal, window, scale, max_len, out, stream
PyObject* do_kv_attention(const Pool& p, const PlanRef& ref, PyObject* const* g)
{
    GBS_BEGIN
    Rows q, o;
    Items it;
    int most, window, longest;
    if (!none(g[9]) || !rows3_of(p, g[0], ref.info.d, &q) || !items_of(p, g[1], g[2], q.n, &it)) Py_RETURN_NONE;
    if (q.n > 0x7fffffff || !int_of(none(g[3]) ? nullptr : g[3], none(g[2]) ? 1 : static_cast<int>(std::max<int64_t>(1, q.n)), &most) || !int_of(g[5], 0, &window) || !int_of(g[7], 0, &longest)) Py_RETURN_NONE;
    const int causal = g[4] ? PyObject_IsTrue(g[4]) : 1;
    const double scale = g[6] ? PyFloat_AsDouble(g[6]) : 0.0;
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    int64_t need;
    if (q.heads > 0x7fffffff || gbs_kv_attention_workspace(ref.plan, &p.cache, static_cast<int>(q.heads), q.n, most, &need) != GBS_OK) Py_RETURN_NONE;
    at::Tensor out;
    if (none(g[8])) {
        out = at::detail::empty_cuda(q.t->sizes(), at::kBFloat16, device_of(p), std::nullopt);
        o = {&out, out.data_ptr(), q.n, q.heads, q.heads * ref.info.d, ref.info.d};
    } else if (!rows3_of(p, g[8], ref.info.d, &o) || o.n != q.n || o.heads != q.heads) Py_RETURN_NONE;
    at::Tensor work = at::detail::empty_cuda({need}, at::kByte, device_of(p), std::nullopt);
    void* wp = work.data_ptr();
    if (gbs_kv_attention(ref.plan, &p.cache, it.seqs, it.cu, static_cast<int>(it.n), q.n, most, longest, q.ptr, q.token, q.head,
                         static_cast<int>(q.heads), static_cast<float>(scale), window, causal ? GBS_KV_CAUSAL : 0, o.ptr, o.token, o.head, wp,
                         need, stream_on(p)) != GBS_OK)
        Py_RETURN_NONE;
    if (!none(g[8])) return Py_NewRef(g[8]);
    return THPVariable_Wrap(std::move(out));
    GBS_END
}

// q, seqs, cu_tokens, groups, max_tokens, causal, scale, max_own, max_prefix, out, stream
PyObject* do_kv_shared_attention(const Pool& p, const PlanRef& ref, PyObject* const* g)
{
    GBS_BEGIN
    Rows q, o;
    Items it;
    int most, longest, prefix;
    const int32_t* groups;
    if (!none(g[10]) || !rows3_of(p, g[0], ref.info.d, &q) || !items_of(p, g[1], g[2], q.n, &it)) Py_RETURN_NONE;
    const int64_t n_groups = none(g[3]) ? 1 : length_of(g[3]) - 1;
    if (n_groups < 1 || n_groups > GBS_KV_MAX_ITEMS || !ints_of(p, g[3], n_groups + 1, &groups)) Py_RETURN_NONE;
    if (q.n > 0x7fffffff || !int_of(none(g[4]) ? nullptr : g[4], none(g[2]) ? 1 : static_cast<int>(std::max<int64_t>(1, q.n)), &most) || !int_of(g[7], 0, &longest) || !int_of(g[8], 0, &prefix)) Py_RETURN_NONE;
    const int causal = g[5] ? PyObject_IsTrue(g[5]) : 1;
    const double scale = g[6] ? PyFloat_AsDouble(g[6]) : 0.0;
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const int n = static_cast<int>(it.n), ng = static_cast<int>(n_groups);
    int64_t need;
    if (q.heads > 0x7fffffff || gbs_kv_shared_attention_workspace(ref.plan, &p.cache, n, q.n, most, ng, prefix, static_cast<int>(q.heads), &need) != GBS_OK) Py_RETURN_NONE;
    at::Tensor out;
    if (none(g[9])) {
        out = at::detail::empty_cuda(q.t->sizes(), at::kBFloat16, device_of(p), std::nullopt);
        o = {&out, out.data_ptr(), q.n, q.heads, q.heads * ref.info.d, ref.info.d};
    } else if (!rows3_of(p, g[9], ref.info.d, &o) || o.n != q.n || o.heads != q.heads) Py_RETURN_NONE;
    at::Tensor work = at::detail::empty_cuda({need}, at::kByte, device_of(p), std::nullopt);
    if (gbs_kv_shared_attention(ref.plan, &p.cache, it.seqs, it.cu, n, q.n, most, groups, ng, longest, prefix, q.ptr, q.token, q.head, static_cast<int>(q.heads),
                                static_cast<float>(scale), causal ? GBS_KV_CAUSAL : 0, o.ptr, o.token, o.head, work.data_ptr(), need, stream_on(p)) != GBS_OK)
        Py_RETURN_NONE;
    if (!none(g[9])) return Py_NewRef(g[9]);
    return THPVariable_Wrap(std::move(out));
    GBS_END
}

// weights of cached tokens: [sequences, KV heads, width] in fp32; *width: what it has, or has to have if it is not 0
bool weights_of(const Pool& p, PyObject* o, float** out, int64_t* width)
{
    const at::Tensor* t = cuda_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 3 || !t->is_contiguous() || t->device().index() != p.device) return false;
    if (t->size(0) != p.cache.n_seqs || t->size(1) != p.cache.n_kv_heads || t->size(2) < 1 || (*width && t->size(2) != *width)) return false;
    *width = t->size(2);
    *out = static_cast<float*>(t->data_ptr());
    return true;
}

// q, mass, seqs, cu_tokens, max_tokens, decay, base, causal, window, scale, stream
PyObject* do_kv_attention_mass(const Pool& p, const PlanRef& ref, PyObject* const* g)
{
    GBS_BEGIN
    Rows q;
    Items it;
    int most, window;
    int64_t width = 0;
    float *mass, *base;
    if (!none(g[10]) || !rows3_of(p, g[0], ref.info.d, &q) || !items_of(p, g[2], g[3], q.n, &it)) Py_RETURN_NONE;
    if (!weights_of(p, g[1], &mass, &width) || !weights_of(p, none(g[6]) ? g[1] : g[6], &base, &width)) Py_RETURN_NONE;
    if (q.n > 0x7fffffff || !int_of(none(g[4]) ? nullptr : g[4], none(g[3]) ? 1 : static_cast<int>(std::max<int64_t>(1, q.n)), &most) || !int_of(g[8], 0, &window)) Py_RETURN_NONE;
    const int causal = g[7] ? PyObject_IsTrue(g[7]) : 1;
    const double decay = g[5] ? PyFloat_AsDouble(g[5]) : 1.0, scale = g[9] ? PyFloat_AsDouble(g[9]) : 0.0;
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const int n = static_cast<int>(it.n);
    int64_t need;
    if (q.heads > 0x7fffffff || gbs_kv_attention_mass_workspace(ref.plan, &p.cache, n, q.n, most, static_cast<int>(q.heads), width, &need) != GBS_OK) Py_RETURN_NONE;
    at::Tensor work = at::detail::empty_cuda({need}, at::kByte, device_of(p), std::nullopt);
    if (gbs_kv_attention_mass(ref.plan, &p.cache, it.seqs, it.cu, n, q.n, most, q.ptr, q.token, q.head, static_cast<int>(q.heads), static_cast<float>(scale),
                              window, causal ? GBS_KV_CAUSAL : 0, base, static_cast<float>(decay), mass, width, work.data_ptr(), need, stream_on(p)) != GBS_OK)
        Py_RETURN_NONE;
    return Py_NewRef(g[1]);
    GBS_END
}

// mass, keep, seqs, recent, first, into, stream
PyObject* do_kv_evict(const Pool& p, const PlanRef& ref, PyObject* const* g)
{
    GBS_BEGIN
    int keep, recent, first;
    int64_t width = 0, need;
    float *mass, *into;
    const int32_t* seqs;
    const int64_t n = none(g[2]) ? p.cache.n_seqs : length_of(g[2]);
    if (!none(g[6]) || n < 0 || n > GBS_KV_MAX_ITEMS || !ints_of(p, g[2], n, &seqs)) Py_RETURN_NONE;
    if (!weights_of(p, g[0], &mass, &width) || !weights_of(p, none(g[5]) ? g[0] : g[5], &into, &width)) Py_RETURN_NONE;
    if (!int_of(g[1], 0, &keep) || !int_of(g[3], 0, &recent) || !int_of(g[4], 0, &first)) Py_RETURN_NONE;
    if (gbs_kv_evict_workspace(ref.plan, &p.cache, static_cast<int>(n), keep, &need) != GBS_OK) Py_RETURN_NONE;
    at::Tensor status = ints(p, n), kept = at::detail::empty_cuda({n, p.cache.n_kv_heads, keep}, at::kInt, device_of(p), std::nullopt);
    at::Tensor work = at::detail::empty_cuda({need}, at::kByte, device_of(p), std::nullopt);
    if (gbs_kv_evict(ref.plan, &p.cache, seqs, static_cast<int>(n), keep, recent, first, mass, into, width, static_cast<int32_t*>(kept.data_ptr()),
                     static_cast<int32_t*>(status.data_ptr()), work.data_ptr(), need, stream_on(p)) != GBS_OK)
        Py_RETURN_NONE;
    PyObject* t = PyTuple_New(2);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(std::move(status)));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(std::move(kept)));
    return t;
    GBS_END
}

PyObject* do_kv_compact(const Pool& p, const PlanRef& ref, PyObject* const* g)       // into, page_map, stream
{
    GBS_BEGIN
    if (!none(g[2])) Py_RETURN_NONE;
    PyObject* other = PyObject_GetAttr(g[0], name_calls);
    if (!other) { PyErr_Clear(); Py_RETURN_NONE; }
    const bool regular = Py_TYPE(other) == pool_type && reinterpret_cast<Pool*>(other)->device == p.device && plan_ref(*reinterpret_cast<Pool*>(other)) &&
                         plan_ref(*reinterpret_cast<Pool*>(other))->info.asymmetric == ref.info.asymmetric;
    const gbs_kv_cache_t into = regular ? reinterpret_cast<Pool*>(other)->cache : gbs_kv_cache_t{};      // the caller's argument keeps its tensors
    Py_DECREF(other);
    const int32_t* given;
    if (!regular || !ints_of(p, g[1], p.cache.n_pages, &given)) Py_RETURN_NONE;
    at::Tensor map, live = ints(p, 1);
    if (!given) map = ints(p, p.cache.n_pages);
    int32_t *mp = given ? const_cast<int32_t*>(given) : static_cast<int32_t*>(map.data_ptr()), *lp = static_cast<int32_t*>(live.data_ptr());
    if (gbs_kv_compact(ref.plan, &p.cache, &into, mp, lp, stream_on(p)) != GBS_OK) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(live));
    GBS_END
}

// A method: the names of its arguments in the class's order, how many must be given, and what to do with them; `on_pool` is for KVCache.
constexpr int MOST_ARGS = 11;
struct Method {
    const char* name;
    int count, required;
    const char* args[MOST_ARGS];
    PyObject* (*call)(const PlanRef&, PyObject* const* given);
    PyObject* (*on_pool)(const Pool&, const PlanRef&, PyObject* const* given) = nullptr;
    bool returns_none = false;
};
constexpr Method KV_EXTEND = {"extend", 3, 0, {"seqs", "counts", "stream"}, nullptr, do_kv_extend};
constexpr Method KV_FORK = {"fork", 3, 2, {"src", "dst", "stream"}, nullptr, do_kv_fork};
constexpr Method KV_FREE = {"free", 2, 1, {"seqs", "stream"}, nullptr, do_kv_free, true};
constexpr Method KV_COMPACT = {"compact", 3, 1, {"into", "page_map", "stream"}, nullptr, do_kv_compact};
constexpr Method KV_APPEND = {"append", 6, 2, {"k", "v", "seqs", "cu_tokens", "stream", "status"}, nullptr, do_kv_append, true};
constexpr Method KV_READ = {"read", 5, 0, {"seqs", "cu_tokens", "n_tokens", "out", "stream"}, nullptr, do_kv_read};
constexpr Method KV_ATTENTION = {"attention", 10, 1, {"q", "seqs", "cu_tokens", "max_tokens", "causal", "window", "scale", "max_len", "out", "stream"},
                                 nullptr, do_kv_attention};
constexpr Method KV_SHARED = {"shared_attention", 11, 1, {"q", "seqs", "cu_tokens", "groups", "max_tokens", "causal", "scale", "max_own", "max_prefix", "out", "stream"},
                              nullptr, do_kv_shared_attention};
constexpr Method KV_MASS = {"attention_mass", 11, 2, {"q", "mass", "seqs", "cu_tokens", "max_tokens", "decay", "base", "causal", "window", "scale", "stream"},
                            nullptr, do_kv_attention_mass};
constexpr Method KV_EVICT = {"evict", 7, 2, {"mass", "keep", "seqs", "recent", "first", "into", "stream"}, nullptr, do_kv_evict};

PyObject* or_none(PyObject* o) { return o ? o : Py_None; }

constexpr Method ROTATE = {"rotate_quantize", 4, 1, {"x", "want_y", "out", "stream"}, [](const PlanRef& r, PyObject* const* g) {
    PyObject* a[5] = {nullptr, g[0], g[1] ? g[1] : Py_False, or_none(g[2]), or_none(g[3])};
    return do_rotate_quantize(r, a);
}};
constexpr Method DEQUANTIZE = {"dequantize", 6, 2, {"codes", "scales", "inverse", "dtype", "out", "stream"}, [](const PlanRef& r, PyObject* const* g) {
    PyObject* a[7] = {nullptr, g[0], g[1], g[2] ? g[2] : Py_False, g[3], or_none(g[4]), or_none(g[5])};
    return do_dequantize(r, a);
}};
constexpr Method MATMUL = {"quantized_matmul", 8, 5, {"codes_x", "scales_x", "plan_w", "codes_w", "scales_w", "dtype", "out", "stream"},
                           [](const PlanRef& r, PyObject* const* g) -> PyObject* {
    PyObject* handle = PyObject_GetAttrString(g[2], "handle");
    if (!handle) { PyErr_Clear(); Py_RETURN_NONE; }
    PyObject* a[9] = {nullptr, g[0], g[1], handle, g[3], g[4], g[5], or_none(g[6]), or_none(g[7])};
    PyObject* out = do_quantized_matmul(r, a);
    Py_DECREF(handle);
    return out;
}};
constexpr Method CLIP = {"clip_error", 5, 2, {"x", "alphas", "want_rows", "err_sum", "stream"}, [](const PlanRef& r, PyObject* const* g) -> PyObject* {
    if ((g[2] && g[2] != Py_False) || (g[3] && g[3] != Py_None)) Py_RETURN_NONE;
    PyObject* a[4] = {nullptr, g[0], g[1], or_none(g[4])};
    return do_clip_error(r, a);
}};

// ---- method(name, function, alloc_outputs): a function of Plan with the regular call in front of it
struct MethodObject {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    const Method* method;
    PyObject* wrapped;
    PyObject* alloc;          // Plan.alloc_outputs, or null where the call allocates without it
};
PyObject* name_alloc = nullptr;

// whether the plan's outputs come from Plan's own alloc_outputs (a subclass or an instance may have another)
bool own_alloc(PyObject* plan, PyObject* alloc)
{
    PyObject* f = PyObject_GetAttr(plan, name_alloc);
    if (!f) { PyErr_Clear(); return false; }
    const bool own = PyMethod_Check(f) && PyMethod_GET_FUNCTION(f) == alloc;
    Py_DECREF(f);
    return own;
}

PyObject* method_call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames)
{
    const MethodObject* o = reinterpret_cast<MethodObject*>(self);
    const Method& M = *o->method;
    const Py_ssize_t n = PyVectorcall_NARGS(nargsf) - 1, nk = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    PyObject* calls = n >= 0 ? PyObject_GetAttr(args[0], name_calls) : nullptr;
    if (!calls) PyErr_Clear();
    PyObject* given[MOST_ARGS] = {nullptr};
    const PlanRef* plan = nullptr;
    if (calls && Py_TYPE(calls) == (M.on_pool ? pool_type : calls_type))
        plan = M.on_pool ? plan_ref(*reinterpret_cast<Pool*>(calls)) : &reinterpret_cast<Calls*>(calls)->ref;
    bool regular = plan && plan->plan && n <= M.count;
    for (Py_ssize_t i = 0; regular && i < n; ++i) given[i] = args[1 + i];
    for (Py_ssize_t k = 0; regular && k < nk; ++k) {
        int at = -1;
        for (int i = 0; i < M.count && at < 0; ++i)
            if (PyUnicode_CompareWithASCIIString(PyTuple_GET_ITEM(kwnames, k), M.args[i]) == 0) at = i;
        regular = at >= 0 && !given[at];
        if (regular) given[at] = args[1 + n + k];
    }
    for (int i = 0; regular && i < M.required; ++i) regular = given[i] != nullptr;
    if (regular && o->alloc) regular = own_alloc(args[0], o->alloc);
    PyObject* out = nullptr;
    if (regular) {
        const PlanRef ref = *plan;                                     // the caller's argument keeps the plan
        out = M.on_pool ? M.on_pool(*reinterpret_cast<Pool*>(calls), ref, given) : M.call(ref, given);
        if (out == Py_None) { Py_DECREF(out); regular = false; }
        else if (out && M.returns_none) { Py_DECREF(out); out = Py_NewRef(Py_None); }
    }
    Py_XDECREF(calls);
    return regular ? out : PyObject_Vectorcall(o->wrapped, args, nargsf, kwnames);
}


PyObject* method_get(PyObject* self, PyObject* obj, PyObject*) { return obj ? PyMethod_New(self, obj) : Py_NewRef(self); }
// name, documentation, signature, module: the wrapped function's
PyObject* method_getattro(PyObject* self, PyObject* name)
{
    PyObject* wrapped = reinterpret_cast<MethodObject*>(self)->wrapped;
    if (PyUnicode_CompareWithASCIIString(name, "__wrapped__") == 0) return Py_NewRef(wrapped);
    if (PyUnicode_CompareWithASCIIString(name, "__class__") == 0 || PyUnicode_CompareWithASCIIString(name, "__call__") == 0)
        return PyObject_GenericGetAttr(self, name);
    return PyObject_GetAttr(wrapped, name);
}
int method_traverse(PyObject* self, visitproc visit, void* arg)
{
    MethodObject* o = reinterpret_cast<MethodObject*>(self);
    Py_VISIT(Py_TYPE(self));
    Py_VISIT(o->wrapped);
    Py_VISIT(o->alloc);
    return 0;
}
int method_clear(PyObject* self)
{
    MethodObject* o = reinterpret_cast<MethodObject*>(self);
    Py_CLEAR(o->wrapped);
    Py_CLEAR(o->alloc);
    return 0;
}
void method_dealloc(PyObject* self)
{
    PyTypeObject* type = Py_TYPE(self);
    PyObject_GC_UnTrack(self);
    method_clear(self);
    type->tp_free(self);
    Py_DECREF(type);
}
PyTypeObject* method_type = nullptr;
const Method* const METHODS[] = {&ROTATE, &DEQUANTIZE, &MATMUL, &CLIP, &KV_EXTEND, &KV_FORK, &KV_FREE, &KV_COMPACT, &KV_APPEND, &KV_READ, &KV_ATTENTION, &KV_SHARED, &KV_MASS, &KV_EVICT};

PyObject* make_method(PyObject*, PyObject* args)
{
    const char* name;
    PyObject *wrapped, *alloc;
    if (!PyArg_ParseTuple(args, "sOO", &name, &wrapped, &alloc)) return nullptr;
    const Method* m = nullptr;
    for (const Method* c : METHODS)
        if (strcmp(name, c->name) == 0) m = c;
    if (!m) { PyErr_Format(PyExc_ValueError, "gbs: no native method '%s'", name); return nullptr; }
    MethodObject* o = reinterpret_cast<MethodObject*>(method_type->tp_alloc(method_type, 0));
    if (!o) return nullptr;
    o->vectorcall = method_call;
    o->method = m;
    o->wrapped = Py_NewRef(wrapped);
    o->alloc = alloc == Py_None ? nullptr : Py_NewRef(alloc);
    return reinterpret_cast<PyObject*>(o);
}

template <class F> PyCFunction cfunc(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)); }

PyMethodDef calls_methods[] = {{"clear", calls_clear, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyType_Slot calls_slots[] = {{Py_tp_init, reinterpret_cast<void*>(calls_init)}, {Py_tp_dealloc, reinterpret_cast<void*>(calls_dealloc)},
                             {Py_tp_new, reinterpret_cast<void*>(PyType_GenericNew)}, {Py_tp_methods, calls_methods}, {0, nullptr}};
PyType_Spec calls_spec = {"paper_2504_13989_b200._native.Calls", sizeof(Calls), 0, Py_TPFLAGS_DEFAULT, calls_slots};

PyType_Slot pool_slots[] = {{Py_tp_init, reinterpret_cast<void*>(pool_init)}, {Py_tp_dealloc, reinterpret_cast<void*>(pool_dealloc)},
                            {Py_tp_new, reinterpret_cast<void*>(PyType_GenericNew)}, {0, nullptr}};
PyType_Spec pool_spec = {"paper_2504_13989_b200._native.Pool", sizeof(Pool), 0, Py_TPFLAGS_DEFAULT, pool_slots};

PyMemberDef method_members[] = {{"__vectorcalloffset__", Py_T_PYSSIZET, offsetof(MethodObject, vectorcall), Py_READONLY, nullptr},
                                {nullptr, 0, 0, 0, nullptr}};
PyType_Slot method_slots[] = {{Py_tp_dealloc, reinterpret_cast<void*>(method_dealloc)}, {Py_tp_traverse, reinterpret_cast<void*>(method_traverse)},
                              {Py_tp_clear, reinterpret_cast<void*>(method_clear)}, {Py_tp_call, reinterpret_cast<void*>(PyVectorcall_Call)},
                              {Py_tp_descr_get, reinterpret_cast<void*>(method_get)}, {Py_tp_getattro, reinterpret_cast<void*>(method_getattro)},
                              {Py_tp_members, method_members}, {0, nullptr}};
PyType_Spec method_spec = {"paper_2504_13989_b200._native.Method", sizeof(MethodObject), 0,
                           Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_GC | Py_TPFLAGS_HAVE_VECTORCALL | Py_TPFLAGS_METHOD_DESCRIPTOR |
                               Py_TPFLAGS_DISALLOW_INSTANTIATION, method_slots};

PyMethodDef methods[] = {{ROTATE.name, cfunc(with_handle<do_rotate_quantize, 5>), METH_FASTCALL, nullptr},
                         {DEQUANTIZE.name, cfunc(with_handle<do_dequantize, 7>), METH_FASTCALL, nullptr},
                         {MATMUL.name, cfunc(with_handle<do_quantized_matmul, 9>), METH_FASTCALL, nullptr},
                         {CLIP.name, cfunc(with_handle<do_clip_error, 4>), METH_FASTCALL, nullptr},
                         {"method", make_method, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    name_calls = PyUnicode_InternFromString("_calls");
    name_alloc = PyUnicode_InternFromString("alloc_outputs");
    calls_type = reinterpret_cast<PyTypeObject*>(PyType_FromSpec(&calls_spec));
    pool_type = reinterpret_cast<PyTypeObject*>(PyType_FromSpec(&pool_spec));
    method_type = reinterpret_cast<PyTypeObject*>(PyType_FromSpec(&method_spec));
    PyObject* m = PyModule_Create(&module);
    if (!name_calls || !name_alloc || !calls_type || !pool_type || !method_type || !m ||
        PyModule_AddObjectRef(m, "Calls", reinterpret_cast<PyObject*>(calls_type)) < 0 ||
        PyModule_AddObjectRef(m, "Pool", reinterpret_cast<PyObject*>(pool_type)) < 0) {
        Py_XDECREF(m);
        return nullptr;
    }
    return m;
}
