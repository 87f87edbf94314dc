"""Thin ctypes binding of libgbs.so (the C ABI declared in include/gbs.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch is used for device memory and streams.  There is no CPU fallback: if the shared
library is missing or a call fails, a GbsError is raised.

Plan's per-call methods go through _native.so (csrc/gbs_torch.cpp), which does the regular call's checks,
allocations and marshalling in C; every other call takes the functions below.  When it is loaded, with the first
plan of a process, its method objects take the place of those methods in the class.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libgbs.so")

GBS_OK = 0
GBS_ERR_INVALID_ARG = -1
GBS_ERR_UNSUPPORTED = -2
GBS_ERR_ALIGNMENT = -3
GBS_ERR_CUDA = -4
GBS_ERR_ALLOC = -5
GBS_DTYPE_F32 = 0
GBS_DTYPE_BF16 = 1
GBS_INVERSE_ROTATE = 1
GBS_MAX_D_PAD = 32768
GBS_MAX_CANDIDATES = 64

GBS_PLAN_ASYMMETRIC = 1

GBS_KV_MAX_ITEMS = 8192
GBS_KV_CAUSAL = 1
GBS_KV_DONE, GBS_KV_BAD_INDEX, GBS_KV_NOT_EMPTY, GBS_KV_NO_PAGES, GBS_KV_TOO_LONG, GBS_KV_DUPLICATE = range(6)
EXPORTS = ("gbs_plan_create", "gbs_plan_create_ex", "gbs_plan_destroy", "gbs_plan_info", "gbs_plan_device_status", "gbs_rotate_quantize",
           "gbs_rotate_quantize_static", "gbs_static_device_status", "gbs_dequantize", "gbs_clip_error",
           "gbs_search_clip_ratio", "gbs_search_state_init", "gbs_search_clip_ratio_fn", "gbs_search_clip_ratio_batch",
           "gbs_hadamard_m", "gbs_status_string", "gbs_selftest_wait_expiry", "gbs_weight_rotate_quantize",
           "gbs_quantized_matmul", "gbs_kv_page_bytes", "gbs_kv_extend", "gbs_kv_fork", "gbs_kv_free", "gbs_kv_compact",
           "gbs_kv_append", "gbs_kv_append_extended", "gbs_kv_read", "gbs_kv_attention_workspace", "gbs_kv_attention",
           "gbs_selftest_kv_attention", "gbs_kv_shared_attention_workspace", "gbs_kv_shared_attention",
           "gbs_kv_attention_mass_workspace", "gbs_kv_attention_mass", "gbs_kv_evict_workspace", "gbs_kv_evict",
           "gbs_selftest_kv_attention_mass", "gbs_selftest_kv_shared_attention")
GBS_STATIC_MAX_D_PAD = 4096


class GbsError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s" % (what, status_string(status)))


class PlanInfo(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int), ("d_pad", ctypes.c_int), ("m", ctypes.c_int), ("k", ctypes.c_int),
                ("bits", ctypes.c_int), ("group", ctypes.c_int), ("alpha", ctypes.c_float),
                ("levels", ctypes.c_int), ("q_lo", ctypes.c_int), ("q_hi", ctypes.c_int),
                ("code_bytes_per_row", ctypes.c_int64), ("scales_per_row", ctypes.c_int),
                ("asymmetric", ctypes.c_int), ("scale_floats_per_row", ctypes.c_int),
                ("variant", ctypes.c_int)]


class SearchResult(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("a", ctypes.c_float), ("b", ctypes.c_float), ("err", ctypes.c_double),
                ("iterations", ctypes.c_int), ("evaluations", ctypes.c_int), ("rounds", ctypes.c_int)]


class SearchState(ctypes.Structure):
    """gbs_search_state_t: the resumable state of one projection's search (plain data; bytes(state) stores it)."""
    _fields_ = [("a", ctypes.c_double), ("b", ctypes.c_double), ("m", ctypes.c_double), ("f_m", ctypes.c_double),
                ("iteration", ctypes.c_int), ("evaluations", ctypes.c_int), ("have_fm", ctypes.c_int),
                ("done", ctypes.c_int)]


class SearchTask(ctypes.Structure):
    _fields_ = [("plan", ctypes.c_void_p), ("x", ctypes.c_void_p), ("x_dtype", ctypes.c_int),
                ("n_rows", ctypes.c_int64), ("x_row_stride", ctypes.c_int64)]


class KVCacheStruct(ctypes.Structure):
    """gbs_kv_cache_t: the arrays and sizes of a pool."""
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("n_kv_heads", ctypes.c_int), ("page_size", ctypes.c_int),
                ("page_table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int), ("max_pages", ctypes.c_int)]


OBJECTIVE_FN = ctypes.CFUNCTYPE(ctypes.c_double, ctypes.c_float, ctypes.c_void_p)
GBS_MAX_SEARCH_TASKS = 4096

_lib = None


def lib() -> ctypes.CDLL:
    """Load libgbs.so (built in-tree by paper_2504_13989_b200.build); fail loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise GbsErrorMissing("libgbs.so not found at %s -- run `python -m paper_2504_13989_b200.build` "
                                  "(or __graft_entry__.build()); there is no CPU fallback" % _LIB_PATH)
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.gbs_plan_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32, i32, ctypes.c_float]
        L.gbs_plan_create.restype = i32
        L.gbs_plan_create_ex.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32, i32, ctypes.c_float, i32]
        L.gbs_plan_create_ex.restype = i32
        L.gbs_plan_destroy.argtypes = [vp]
        L.gbs_plan_destroy.restype = i32
        L.gbs_plan_info.argtypes = [vp, ctypes.POINTER(PlanInfo)]
        L.gbs_plan_info.restype = i32
        L.gbs_plan_device_status.argtypes = [vp, ctypes.POINTER(i32)]
        L.gbs_plan_device_status.restype = i32
        L.gbs_rotate_quantize.argtypes = [vp, vp, i32, i64, i64, vp, vp, vp, vp]
        L.gbs_rotate_quantize.restype = i32
        L.gbs_rotate_quantize_static.argtypes = [i32, i32, i32, i32, i32, ctypes.c_float, vp, i64, i64, vp, vp, vp]
        L.gbs_rotate_quantize_static.restype = i32
        L.gbs_selftest_wait_expiry.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.gbs_selftest_wait_expiry.restype = i32
        L.gbs_static_device_status.argtypes = [ctypes.POINTER(i32)]
        L.gbs_static_device_status.restype = i32
        L.gbs_dequantize.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp]
        L.gbs_dequantize.restype = i32
        L.gbs_clip_error.argtypes = [vp, vp, i32, i64, i64, ctypes.POINTER(ctypes.c_float), i32, vp, vp, vp]
        L.gbs_clip_error.restype = i32
        L.gbs_search_clip_ratio.argtypes = [vp, vp, i32, i64, i64, ctypes.c_float, vp, ctypes.POINTER(SearchResult), vp]
        L.gbs_search_clip_ratio.restype = i32
        L.gbs_search_state_init.argtypes = [ctypes.POINTER(SearchState)]
        L.gbs_search_state_init.restype = i32
        L.gbs_search_clip_ratio_fn.argtypes = [OBJECTIVE_FN, vp, ctypes.c_float, ctypes.POINTER(SearchState), i32]
        L.gbs_search_clip_ratio_fn.restype = i32
        L.gbs_search_clip_ratio_batch.argtypes = [ctypes.POINTER(SearchTask), i32, ctypes.c_float,
                                                  ctypes.POINTER(SearchState), i32, vp, ctypes.POINTER(ctypes.c_float),
                                                  ctypes.POINTER(i32), vp]
        L.gbs_search_clip_ratio_batch.restype = i32
        L.gbs_weight_rotate_quantize.argtypes = [vp, vp, i32, i64, i64, vp, vp, vp]
        L.gbs_weight_rotate_quantize.restype = i32
        L.gbs_quantized_matmul.argtypes = [vp, vp, vp, i64, vp, vp, vp, i64, vp, i32, i64, vp]
        L.gbs_quantized_matmul.restype = i32
        kv = ctypes.POINTER(KVCacheStruct)
        L.gbs_kv_page_bytes.argtypes = [vp, i32, i32, ctypes.POINTER(i64)]
        L.gbs_kv_extend.argtypes = [vp, kv, vp, vp, i32, vp, vp]
        L.gbs_kv_fork.argtypes = [vp, kv, vp, vp, i32, vp, vp]
        L.gbs_kv_free.argtypes = [vp, kv, vp, i32, vp]
        L.gbs_kv_compact.argtypes = [vp, kv, kv, vp, vp, vp]
        L.gbs_kv_append.argtypes = [vp, kv, vp, vp, i32, i64, vp, vp, i64, i64, vp]
        L.gbs_kv_append_extended.argtypes = [vp, kv, vp, vp, i32, i64, vp, vp, i64, i64, vp, vp]
        L.gbs_kv_read.argtypes = [vp, kv, vp, vp, i32, i64, vp, vp, vp]
        L.gbs_kv_attention_workspace.argtypes = [vp, kv, i32, i64, i32, ctypes.POINTER(i64)]
        L.gbs_kv_attention.argtypes = [vp, kv, vp, vp, i32, i64, i32, i32, vp, i64, i64, i32, ctypes.c_float, i32, i32, vp, i64, i64,
                                       vp, i64, vp]
        L.gbs_selftest_kv_attention.argtypes = L.gbs_kv_attention.argtypes[:-1] + [i32, i32, vp]
        L.gbs_kv_shared_attention_workspace.argtypes = [vp, kv, i32, i64, i32, i32, i32, i32, ctypes.POINTER(i64)]
        L.gbs_kv_shared_attention.argtypes = [vp, kv, vp, vp, i32, i64, i32, vp, i32, i32, i32, vp, i64, i64, i32, ctypes.c_float, i32, vp, i64, i64,
                                              vp, i64, vp]
        L.gbs_selftest_kv_shared_attention.argtypes = L.gbs_kv_shared_attention.argtypes[:-1] + [i32, i32, vp]
        L.gbs_kv_attention_mass_workspace.argtypes = [vp, kv, i32, i64, i32, i32, i64, ctypes.POINTER(i64)]
        L.gbs_kv_attention_mass.argtypes = [vp, kv, vp, vp, i32, i64, i32, vp, i64, i64, i32, ctypes.c_float, i32, i32, vp, ctypes.c_float, vp, i64,
                                            vp, i64, vp]
        L.gbs_selftest_kv_attention_mass.argtypes = L.gbs_kv_attention_mass.argtypes[:-1] + [i32, i32, vp]
        L.gbs_kv_evict_workspace.argtypes = [vp, kv, i32, i32, ctypes.POINTER(i64)]
        L.gbs_kv_evict.argtypes = [vp, kv, vp, i32, i32, i32, i32, vp, vp, i64, vp, vp, vp, i64, vp]
        for name in EXPORTS[EXPORTS.index("gbs_kv_page_bytes"):]:
            getattr(L, name).restype = i32
        L.gbs_hadamard_m.argtypes = [i32, vp]
        L.gbs_hadamard_m.restype = i32
        L.gbs_status_string.argtypes = [i32]
        L.gbs_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


_native_module = None


def native():
    """Load _native.so (built beside libgbs.so); fail loudly if absent."""
    global _native_module
    if _native_module is None:
        lib()
        try:
            from . import _native
        except ImportError as e:
            raise GbsErrorMissing("_native.so does not load (%s) -- run `python -m paper_2504_13989_b200.build`" % e) from e
        for name, f in _PYTHON_METHODS.items():
            if Plan.__dict__.get(name) is f:                      # a method that was replaced stays
                setattr(Plan, name, _native.method(name, f, Plan.alloc_outputs if name == "rotate_quantize" else None))
        for name, f in _PYTHON_KV_METHODS.items():
            if KVCache.__dict__.get(name) is f:
                setattr(KVCache, name, _native.method(name, f, None))
        _native_module = _native
    return _native_module


class GbsErrorMissing(RuntimeError):
    pass


def status_string(status: int) -> str:
    return lib().gbs_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != GBS_OK:
        raise GbsError(status, what)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GBS_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return GBS_DTYPE_BF16
    raise TypeError("gbs: tensors must be float32 or bfloat16, got %s" % t.dtype)


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _rows_view(x: torch.Tensor, d: int):
    """(pointer, n_rows, row stride in elements) of a [..., d] tensor whose leading dims are contiguous rows."""
    if not x.is_cuda:
        raise ValueError("gbs: x must be a CUDA tensor (device pointer); there is no CPU path")
    if x.dim() < 1 or x.shape[-1] != d:
        raise ValueError("gbs: last dimension of x must be d=%d, got shape %s" % (d, tuple(x.shape)))
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if x.stride(-1) != 1:
        raise ValueError("gbs: the last dimension of x must be contiguous")
    if x.dim() > 2:
        x = x.reshape(-1, d) if x.is_contiguous() else x.flatten(0, -2)
    return x, x.shape[0], (x.stride(0) if x.shape[0] > 1 else max(x.stride(0), d))


def _check_buffer(what: str, t: torch.Tensor, like: torch.Tensor, dtype, min_numel: int):
    """The C ABI cannot validate pointers; the binding knows the tensors behind them.  An undersized, CPU or
    strided buffer would make a kernel write out of bounds on the device, so it is refused here."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("gbs: %s must be a CUDA tensor" % what)
    if t.device != like.device:
        raise ValueError("gbs: %s is on %s but the rows are on %s" % (what, t.device, like.device))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("gbs: %s must be %s, got %s" % (what, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("gbs: %s must be contiguous" % what)
    if t.numel() < min_numel:
        raise ValueError("gbs: %s holds %d elements, the call writes %d" % (what, t.numel(), min_numel))


# ----------------------------------------------------------------------------------------------
# functions named after the C entry points
# ----------------------------------------------------------------------------------------------
def gbs_plan_create(d: int, d_pad: int, m: int, bits: int, group: int, alpha: float) -> int:
    """Returns an opaque plan handle (int).  See include/gbs.h for the argument ranges."""
    h = ctypes.c_void_p()
    _check(lib().gbs_plan_create(ctypes.byref(h), d, d_pad, m, bits, group, alpha), "gbs_plan_create")
    return h.value


def gbs_plan_create_ex(d: int, d_pad: int, m: int, bits: int, group: int, alpha: float, flags: int) -> int:
    """gbs_plan_create with flags (GBS_PLAN_ASYMMETRIC: the asymmetric quantizer for d' = 128 KV rows)."""
    h = ctypes.c_void_p()
    _check(lib().gbs_plan_create_ex(ctypes.byref(h), d, d_pad, m, bits, group, alpha, flags), "gbs_plan_create_ex")
    return h.value


def gbs_plan_destroy(plan: int) -> None:
    _check(lib().gbs_plan_destroy(ctypes.c_void_p(plan)), "gbs_plan_destroy")


def gbs_plan_info(plan: int) -> PlanInfo:
    info = PlanInfo()
    _check(lib().gbs_plan_info(ctypes.c_void_p(plan), ctypes.byref(info)), "gbs_plan_info")
    return info


def gbs_plan_device_status(plan: int) -> int:
    """Read and clear the plan's device status word (0 = no bounded wait ever expired).  Synchronises."""
    v = ctypes.c_int(0)
    _check(lib().gbs_plan_device_status(ctypes.c_void_p(plan), ctypes.byref(v)), "gbs_plan_device_status")
    return v.value


def gbs_hadamard_m(m: int) -> torch.Tensor:
    """The m x m sign matrix H_m the plans use (host computation, int8)."""
    out = torch.zeros((m, m), dtype=torch.int8)
    _check(lib().gbs_hadamard_m(m, out.data_ptr()), "gbs_hadamard_m")
    return out


def gbs_rotate_quantize(plan: int, x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                        y_opt: torch.Tensor | None = None, stream=None) -> None:
    info = gbs_plan_info(plan)
    xv, n_rows, stride = _rows_view(x, info.d)
    _check_buffer("codes", codes, xv, torch.uint8, n_rows * info.code_bytes_per_row)
    _check_buffer("scales", scales, xv, torch.float32, n_rows * info.scale_floats_per_row)
    if y_opt is not None:
        _check_buffer("y_opt", y_opt, xv, torch.float32, n_rows * info.d_pad)
    _check(lib().gbs_rotate_quantize(ctypes.c_void_p(plan), xv.data_ptr(), _dtype_code(xv), n_rows, stride,
                                     codes.data_ptr(), scales.data_ptr(),
                                     y_opt.data_ptr() if y_opt is not None else None, _stream_ptr(stream)),
           "gbs_rotate_quantize")


def gbs_rotate_quantize_static(d: int, d_pad: int, m: int, bits: int, group: int, alpha: float, x: torch.Tensor,
                               codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """gbs_rotate_quantize without a plan and without any device allocation inside the library: for
    processes that may not call cudaMalloc (all memory already claimed by a pool, or no tolerance for
    the device-wide synchronisation an allocation implies).  bf16 rows, d_pad <= GBS_STATIC_MAX_D_PAD;
    see include/gbs.h for the limits and for how calls share the library's fixed device array."""
    xv, n_rows, stride = _rows_view(x, d)
    if xv.dtype != torch.bfloat16:
        raise TypeError("gbs_rotate_quantize_static: x must be bfloat16")
    if d_pad > 0 and bits in (3, 4):
        _check_buffer("codes", codes, xv, torch.uint8, n_rows * (d_pad * bits // 8))
        _check_buffer("scales", scales, xv, torch.float32, n_rows * (d_pad // group if group > 0 else 1))
    _check(lib().gbs_rotate_quantize_static(d, d_pad, m, bits, group, alpha, xv.data_ptr(), n_rows, stride,
                                            codes.data_ptr(), scales.data_ptr(), _stream_ptr(stream)),
           "gbs_rotate_quantize_static")


def gbs_selftest_wait_expiry(limit_us: int = 1000):
    """Run one bounded wait that is certain to run out; returns (code, abort flag, microseconds waited)."""
    code, ab, us = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().gbs_selftest_wait_expiry(int(limit_us), ctypes.byref(code), ctypes.byref(ab), ctypes.byref(us)),
           "gbs_selftest_wait_expiry")
    return code.value, ab.value, us.value


def gbs_static_device_status() -> int:
    """Read and clear the status word of gbs_rotate_quantize_static on the current device.  Synchronises."""
    v = ctypes.c_int(0)
    _check(lib().gbs_static_device_status(ctypes.byref(v)), "gbs_static_device_status")
    return v.value


def gbs_dequantize(plan: int, codes: torch.Tensor, scales: torch.Tensor, n_rows: int, out: torch.Tensor,
                   flags: int = 0, stream=None) -> None:
    info = gbs_plan_info(plan)
    width = info.d if (flags & GBS_INVERSE_ROTATE) else info.d_pad
    _check_buffer("codes", codes, codes, torch.uint8, n_rows * info.code_bytes_per_row)
    _check_buffer("scales", scales, codes, torch.float32, n_rows * info.scale_floats_per_row)
    _check_buffer("out", out, codes, None, n_rows * width)
    _check(lib().gbs_dequantize(ctypes.c_void_p(plan), codes.data_ptr(), scales.data_ptr(), n_rows,
                                out.data_ptr(), _dtype_code(out), flags, _stream_ptr(stream)),
           "gbs_dequantize")


def gbs_clip_error(plan: int, x: torch.Tensor, alphas, err_sum: torch.Tensor,
                   err_rows_opt: torch.Tensor | None = None, stream=None) -> None:
    info = gbs_plan_info(plan)
    xv, n_rows, stride = _rows_view(x, info.d)
    alphas = [float(a) for a in alphas]
    arr = (ctypes.c_float * len(alphas))(*alphas)
    _check_buffer("err_sum", err_sum, xv, torch.float64, len(alphas))
    if err_rows_opt is not None:
        _check_buffer("err_rows_opt", err_rows_opt, xv, torch.float32, n_rows * len(alphas))
    _check(lib().gbs_clip_error(ctypes.c_void_p(plan), xv.data_ptr(), _dtype_code(xv), n_rows, stride,
                                arr, len(alphas), err_sum.data_ptr(),
                                err_rows_opt.data_ptr() if err_rows_opt is not None else None,
                                _stream_ptr(stream)),
           "gbs_clip_error")


def gbs_search_clip_ratio(plan: int, x: torch.Tensor, eps: float, work: torch.Tensor | None = None,
                          stream=None) -> SearchResult:
    """Algorithm 1's bracket search for the clip ratio of the rows in x (objective: quantization error).
    Blocks on the stream after every round of up to 31 probes."""
    info = gbs_plan_info(plan)
    xv, n_rows, stride = _rows_view(x, info.d)
    if work is None:
        work = torch.empty(GBS_MAX_CANDIDATES, dtype=torch.float64, device=x.device)
    _check_buffer("work", work, xv, torch.float64, GBS_MAX_CANDIDATES)
    res = SearchResult()
    _check(lib().gbs_search_clip_ratio(ctypes.c_void_p(plan), xv.data_ptr(), _dtype_code(xv), n_rows, stride,
                                       float(eps), work.data_ptr(), ctypes.byref(res), _stream_ptr(stream)),
           "gbs_search_clip_ratio")
    return res


def gbs_weight_rotate_quantize(plan: int, w: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """Rows of the weight matrix [n_out, d] through the activation path's rotation and quantizer (Eq. (2))."""
    info = gbs_plan_info(plan)
    wv, n_out, stride = _rows_view(w, info.d)
    _check_buffer("codes", codes, wv, torch.uint8, n_out * info.code_bytes_per_row)
    _check_buffer("scales", scales, wv, torch.float32, n_out * info.scale_floats_per_row)
    _check(lib().gbs_weight_rotate_quantize(ctypes.c_void_p(plan), wv.data_ptr(), _dtype_code(wv), n_out, stride,
                                            codes.data_ptr(), scales.data_ptr(), _stream_ptr(stream)),
           "gbs_weight_rotate_quantize")


def gbs_quantized_matmul(plan_x: int, codes_x: torch.Tensor, scales_x: torch.Tensor, plan_w: int, codes_w: torch.Tensor,
                         scales_w: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """out[t, o] = Delta_x[t] * Delta_w[o] * sum_j q_x[t, j] * q_w[o, j] from the packed codes of both sides."""
    ix, iw = gbs_plan_info(plan_x), gbs_plan_info(plan_w)
    n_tok, n_out = codes_x.shape[0], codes_w.shape[0]
    _check_buffer("codes_x", codes_x, codes_x, torch.uint8, n_tok * ix.code_bytes_per_row)
    _check_buffer("scales_x", scales_x, codes_x, torch.float32, n_tok * ix.scale_floats_per_row)
    _check_buffer("codes_w", codes_w, codes_x, torch.uint8, n_out * iw.code_bytes_per_row)
    _check_buffer("scales_w", scales_w, codes_x, torch.float32, n_out * iw.scale_floats_per_row)
    if out.dim() != 2 or out.shape[0] != n_tok or out.shape[1] != n_out or out.stride(1) != 1 or not out.is_cuda \
            or out.device != codes_x.device:
        raise ValueError("gbs_quantized_matmul: out must be a CUDA [n_tokens, n_out] tensor with contiguous rows")
    _check(lib().gbs_quantized_matmul(ctypes.c_void_p(plan_x), codes_x.data_ptr(), scales_x.data_ptr(), n_tok,
                                      ctypes.c_void_p(plan_w), codes_w.data_ptr(), scales_w.data_ptr(), n_out,
                                      out.data_ptr(), _dtype_code(out), out.stride(0), _stream_ptr(stream)),
           "gbs_quantized_matmul")


def gbs_search_state_init() -> SearchState:
    st = SearchState()
    _check(lib().gbs_search_state_init(ctypes.byref(st)), "gbs_search_state_init")
    return st


def gbs_search_clip_ratio_fn(objective, eps: float, state: SearchState | None = None,
                             max_iterations: int = 0) -> SearchState:
    """Algorithm 1's loop for one projection with a Python objective `objective(alpha) -> float` (e.g. a model's
    perplexity).  Host only.  Returns the state (done = 1 when b - a <= eps); pass it back to resume."""
    st = state if state is not None else gbs_search_state_init()
    cb = OBJECTIVE_FN(lambda alpha, _ctx: float(objective(float(alpha))))
    _check(lib().gbs_search_clip_ratio_fn(cb, None, float(eps), ctypes.byref(st), int(max_iterations)),
           "gbs_search_clip_ratio_fn")
    return st


def gbs_search_clip_ratio_batch(plans, xs, eps: float, states=None, max_rounds: int = 0, work: torch.Tensor | None = None,
                                stream=None):
    """Algorithm 1's loop for several projections at once (plan i scores rows xs[i]); one wait per round.
    Returns (alphas: the list L, states, rounds).  `plans` are plan handles (ints)."""
    n = len(plans)
    if n < 1 or n != len(xs):
        raise ValueError("gbs_search_clip_ratio_batch: one tensor per plan")
    tasks = (SearchTask * n)()
    keep = []
    for i, (pl, x) in enumerate(zip(plans, xs)):
        info = gbs_plan_info(pl)
        xv, n_rows, stride = _rows_view(x, info.d)
        keep.append(xv)
        tasks[i] = SearchTask(pl, xv.data_ptr(), _dtype_code(xv), n_rows, stride)
    sts = (SearchState * n)()
    for i in range(n):
        sts[i] = states[i] if states is not None else gbs_search_state_init()
    if work is None:
        work = torch.empty(n * GBS_MAX_CANDIDATES, dtype=torch.float64, device=keep[0].device)
    _check_buffer("work", work, keep[0], torch.float64, n * GBS_MAX_CANDIDATES)
    alphas = (ctypes.c_float * n)()
    rounds = ctypes.c_int(0)
    _check(lib().gbs_search_clip_ratio_batch(tasks, n, float(eps), sts, int(max_rounds), work.data_ptr(), alphas,
                                             ctypes.byref(rounds), _stream_ptr(stream)),
           "gbs_search_clip_ratio_batch")
    return [float(a) for a in alphas], [sts[i] for i in range(n)], rounds.value


# ----------------------------------------------------------------------------------------------
# convenience object: owns a plan handle and allocates outputs with torch
# ----------------------------------------------------------------------------------------------
class Plan:
    """RAII wrapper of a gbs plan; allocates output tensors with torch and forwards to the C ABI."""

    def __init__(self, d: int, d_pad: int | None = None, m: int = 1, bits: int = 4, group: int = 0,
                 alpha: float = 1.0, asymmetric: bool = False):
        d_pad = d if d_pad is None else d_pad
        calls = native().Calls
        self.handle = gbs_plan_create_ex(d, d_pad, m, bits, group, alpha, GBS_PLAN_ASYMMETRIC if asymmetric else 0)
        self.info = gbs_plan_info(self.handle)
        self._device = torch.cuda.current_device()                 # the plan's, since the C call takes the current one
        self._calls = calls(self.handle)                           # what the native methods know of this plan

    def close(self):
        if getattr(self, "handle", None):
            self._calls.clear()
            gbs_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def device_status(self) -> int:
        return gbs_plan_device_status(self.handle)

    def alloc_outputs(self, n_rows: int, device, want_y: bool = False):
        codes = torch.empty((n_rows, self.info.code_bytes_per_row), dtype=torch.uint8, device=device)
        scales = torch.empty((n_rows, self.info.scale_floats_per_row), dtype=torch.float32, device=device)
        y = torch.empty((n_rows, self.info.d_pad), dtype=torch.float32, device=device) if want_y else None
        return codes, scales, y

    def rotate_quantize(self, x: torch.Tensor, want_y: bool = False, out=None, stream=None):
        n_rows = x.numel() // self.info.d
        codes, scales, y = out if out is not None else self.alloc_outputs(n_rows, x.device, want_y)
        gbs_rotate_quantize(self.handle, x, codes, scales, y, stream)
        return codes, scales, y

    def dequantize(self, codes: torch.Tensor, scales: torch.Tensor, inverse: bool = False,
                   dtype=torch.float32, out=None, stream=None) -> torch.Tensor:
        n_rows = codes.shape[0]
        width = self.info.d if inverse else self.info.d_pad
        if out is None:
            out = torch.empty((n_rows, width), dtype=dtype, device=codes.device)
        gbs_dequantize(self.handle, codes, scales, n_rows, out, GBS_INVERSE_ROTATE if inverse else 0, stream)
        return out

    def clip_error(self, x: torch.Tensor, alphas, want_rows: bool = False, err_sum=None, stream=None):
        n_rows = x.numel() // self.info.d
        K = len(alphas)
        if err_sum is None:
            err_sum = torch.zeros(K, dtype=torch.float64, device=x.device)
        rows = torch.empty((n_rows, K), dtype=torch.float32, device=x.device) if want_rows else None
        gbs_clip_error(self.handle, x, alphas, err_sum, rows, stream)
        return (err_sum, rows) if want_rows else err_sum

    def weight_rotate_quantize(self, w: torch.Tensor, out=None, stream=None):
        """Quantize the rows of a weight matrix [n_out, d] (Eq. (2)); returns (codes, scales)."""
        n_out = w.numel() // self.info.d
        codes, scales, _ = out if out is not None else self.alloc_outputs(n_out, w.device)
        gbs_weight_rotate_quantize(self.handle, w, codes, scales, stream)
        return codes, scales

    def quantized_matmul(self, codes_x, scales_x, plan_w: "Plan", codes_w, scales_w, dtype=torch.float32, out=None,
                         stream=None) -> torch.Tensor:
        """The layer's output from the packed codes of activations (this plan) and weights (plan_w)."""
        if out is None:
            out = torch.empty((codes_x.shape[0], codes_w.shape[0]), dtype=dtype, device=codes_x.device)
        gbs_quantized_matmul(self.handle, codes_x, scales_x, plan_w.handle, codes_w, scales_w, out, stream)
        return out

    def search_clip_ratio(self, x: torch.Tensor, eps: float = 1.0 / 64, stream=None) -> SearchResult:
        return gbs_search_clip_ratio(self.handle, x, eps, stream=stream)

    def rotate_quantize_host(self, x_host: torch.Tensor, codes_host: torch.Tensor, scales_host: torch.Tensor,
                             device="cuda:0", stream=None):
        """End-to-end call for host-resident data: pinned host -> device, rotate_quantize, device -> host.

        x_host / codes_host / scales_host are (ideally pinned) CPU tensors; the copies are enqueued on
        the same stream as the kernel.  Returns after the stream has been synchronised.
        """
        s = stream or torch.cuda.current_stream()
        with torch.cuda.stream(s):
            x = x_host.to(device, non_blocking=True)
            codes, scales, _ = self.rotate_quantize(x, stream=s)
            codes_host.copy_(codes, non_blocking=True)
            scales_host.copy_(scales, non_blocking=True)
        s.synchronize()
        return codes_host, scales_host


# ----------------------------------------------------------------------------------------------
# paged KV cache in four bits
# ----------------------------------------------------------------------------------------------
def _int32(what: str, v: int) -> int:
    """ctypes would cut a larger number to 32 bits."""
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError("gbs: %s does not fit 32 bits: %d" % (what, v))
    return v


def gbs_kv_page_bytes(plan: int, n_kv_heads: int, page_size: int) -> int:
    """Bytes of one page of a pool (host only)."""
    _int32("n_kv_heads", n_kv_heads), _int32("page_size", page_size)
    out = ctypes.c_int64(0)
    _check(lib().gbs_kv_page_bytes(ctypes.c_void_p(plan), n_kv_heads, page_size, ctypes.byref(out)), "gbs_kv_page_bytes")
    return out.value


class KVCache:
    """A pool of pages that holds rotated, quantized keys and values, and the calls on it (gbs_kv_* in include/gbs.h).

    The tensors belong to the caller and are used in place: pages [n_pages, gbs_kv_page_bytes] uint8, page_table
    [n_seqs, max_pages], lengths [n_seqs] and refs [n_pages] int32.  KVCache.create makes them, empty.  Items of a call are
    sequences: `seqs` (int32, None: 0, 1, ..), with `cu_tokens` (int32, [items + 1]) where an item has other than one token; their
    tokens are the last ones of the sequences.  Nothing here waits for the device: what became of the items of extend and fork
    stands in the tensors these return.  With `stream`, a call's results are
    allocated on it; ordering it behind the work that its arguments come from is the caller's.
    """

    def __init__(self, plan: Plan, pages: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor,
                 n_kv_heads: int, page_size: int):
        self.page_bytes = gbs_kv_page_bytes(plan.handle, n_kv_heads, page_size)
        for what, t, dtype, shape in (("pages", pages, torch.uint8, (pages.shape[0], self.page_bytes)),
                                      ("page_table", page_table, torch.int32, tuple(page_table.shape[:2])),
                                      ("lengths", lengths, torch.int32, tuple(page_table.shape[:1])),
                                      ("refs", refs, torch.int32, tuple(pages.shape[:1]))):
            _check_buffer(what, t, pages, dtype, 1)
            if tuple(t.shape) != shape:
                raise ValueError("gbs: %s must have shape %s, got %s" % (what, shape, tuple(t.shape)))
        if page_table.dim() != 2:
            raise ValueError("gbs: page_table must be [sequences, pages]")
        if pages.device.index != plan._device:
            raise ValueError("gbs: the pool is on %s, its plan on cuda:%d" % (pages.device, plan._device))
        self.plan, self.n_kv_heads, self.page_size = plan, n_kv_heads, page_size
        self.pages, self.page_table, self.lengths, self.refs = pages, page_table, lengths, refs
        self._kept = pages, page_table, lengths, refs              # the calls use these, whatever the names above are bound to later
        self._c = KVCacheStruct(pages.data_ptr(), pages.shape[0], n_kv_heads, page_size, page_table.data_ptr(), lengths.data_ptr(),
                                refs.data_ptr(), page_table.shape[0], page_table.shape[1])
        self._calls = native().Pool(plan._calls, pages, page_table, lengths, refs, n_kv_heads, page_size)

    @classmethod
    def create(cls, plan: Plan, n_pages: int, n_kv_heads: int, page_size: int, n_seqs: int, max_pages: int, device="cuda:0"):
        """An empty pool."""
        pages = torch.empty((n_pages, gbs_kv_page_bytes(plan.handle, n_kv_heads, page_size)), dtype=torch.uint8, device=device)
        table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device)
        return cls(plan, pages, table, torch.zeros(n_seqs, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device), n_kv_heads, page_size)

    def _empty(self, stream, shape, dtype, handed_on=True):
        """Memory for a call's results or its workspace, taken on the call's stream: a block that is free on another one may still be used by
        work that waits there.  Results, which the caller's stream goes on with, are not taken again before that one is done with them."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.pages.device)
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=self.pages.device)
        if handed_on:
            t.record_stream(torch.cuda.current_stream(self.pages.device))
        return t

    def _stream(self, stream, *used):
        """The call's stream; the tensors that it uses are kept until it is done with them, whichever stream they are freed on."""
        if stream is None:
            return int(torch.cuda.current_stream(self.pages.device).cuda_stream)
        if stream.device != self.pages.device:
            raise ValueError("gbs: the pool is on %s, the stream on %s" % (self.pages.device, stream.device))
        for t in self._kept + used:
            if t is not None:
                t.record_stream(stream)
        return int(stream.cuda_stream)

    def _ints(self, what: str, t, n: int):
        """Pointer of a row of n int32 (None: null)."""
        if t is None:
            return None
        _check_buffer(what, t, self.pages, torch.int32, 0)
        if t.dim() != 1 or t.shape[0] != n:
            raise ValueError("gbs: %s must be one row of %d numbers, got shape %s" % (what, n, tuple(t.shape)))
        return t.data_ptr()

    def _items(self, seqs, cu_tokens, n_tokens: int):
        """(pointer of seqs, pointer of cu_tokens, number of items)"""
        n = seqs.shape[0] if seqs is not None else (cu_tokens.shape[0] - 1 if cu_tokens is not None else n_tokens)
        return self._ints("seqs", seqs, n), self._ints("cu_tokens", cu_tokens, n + 1), n

    def _rows(self, what: str, x: torch.Tensor, heads: int):
        if not isinstance(x, torch.Tensor) or not x.is_cuda or x.device != self.pages.device:
            raise ValueError("gbs: %s must be a tensor on %s" % (what, self.pages.device))
        if x.dtype != torch.bfloat16:
            raise TypeError("gbs: %s must be bfloat16, got %s" % (what, x.dtype))
        d = self.plan.info.d
        if x.dim() != 3 or x.shape[1] != heads or x.shape[2] != d or x.stride(2) != 1:
            raise ValueError("gbs: %s must be [tokens, %d, %d] with contiguous rows, got shape %s, strides %s" %
                             (what, heads, d, tuple(x.shape), x.stride()))

    def _strides(self, x: torch.Tensor):
        # a stride that no element depends on may be anything
        d = self.plan.info.d
        return (x.stride(0) if x.shape[0] > 1 else d), (x.stride(1) if x.shape[1] > 1 else d)

    def extend(self, seqs=None, counts=None, stream=None) -> torch.Tensor:
        """Room for counts[i] (None: one) more tokens in each sequence; returns the items' status (GBS_KV_*)."""
        n = next((t.shape[0] for t in (seqs, counts) if t is not None), self.page_table.shape[0])
        status = self._empty(stream, n, torch.int32)
        _check(lib().gbs_kv_extend(self.plan.handle, ctypes.byref(self._c), self._ints("seqs", seqs, n), self._ints("counts", counts, n), n,
                                   status.data_ptr(), self._stream(stream, seqs, counts)), "gbs_kv_extend")
        return status

    def fork(self, src: torch.Tensor, dst: torch.Tensor, stream=None) -> torch.Tensor:
        """Empty sequences dst[i] become copies of src[i] that share its full pages; returns the pairs' status (GBS_KV_*)."""
        n = src.shape[0]
        status = self._empty(stream, n, torch.int32)
        _check(lib().gbs_kv_fork(self.plan.handle, ctypes.byref(self._c), self._ints("src", src, n), self._ints("dst", dst, n), n,
                                 status.data_ptr(), self._stream(stream, src, dst)), "gbs_kv_fork")
        return status

    def free(self, seqs: torch.Tensor, stream=None) -> None:
        """The sequences end; pages that no other sequence holds are free."""
        _check(lib().gbs_kv_free(self.plan.handle, ctypes.byref(self._c), self._ints("seqs", seqs, seqs.shape[0]), seqs.shape[0],
                                 self._stream(stream, seqs)), "gbs_kv_free")

    def compact(self, into: "KVCache", page_map: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Move the pages in use into the pool `into`, in order; returns their number (one int32 on the device)."""
        if page_map is None:
            page_map = self._empty(stream, self.pages.shape[0], torch.int32, False)
        live = self._empty(stream, 1, torch.int32)
        if into.pages.device != self.pages.device or into.plan.info.asymmetric != self.plan.info.asymmetric:
            raise ValueError("gbs: both pools must be on one device and of one kind of quantizer")
        _check(lib().gbs_kv_compact(self.plan.handle, ctypes.byref(self._c), ctypes.byref(into._c),
                                    self._ints("page_map", page_map, self.pages.shape[0]), live.data_ptr(),
                                    self._stream(stream, page_map, *into._kept)), "gbs_kv_compact")
        return live

    def append(self, k: torch.Tensor, v: torch.Tensor, seqs=None, cu_tokens=None, stream=None, status=None) -> None:
        """Rotate and quantize key and value rows [tokens, n_kv_heads, d] (bf16) into the pages of their tokens.  status: what extend returned
        for these items; those that it refused are left out (without it their rows replace the last ones of their sequences)."""
        self._rows("k", k, self.n_kv_heads)
        self._rows("v", v, self.n_kv_heads)
        if v.shape[0] != k.shape[0]:
            raise ValueError("gbs: k has %d tokens, v %d" % (k.shape[0], v.shape[0]))
        if self._strides(v) != self._strides(k):
            raise ValueError("gbs: k and v must have the same strides, got %s and %s" % (k.stride(), v.stride()))
        s, cu, n = self._items(seqs, cu_tokens, k.shape[0])
        _check(lib().gbs_kv_append_extended(self.plan.handle, ctypes.byref(self._c), s, cu, n, k.shape[0], k.data_ptr(), v.data_ptr(),
                                            *self._strides(k), self._ints("status", status, n),
                                            self._stream(stream, k, v, seqs, cu_tokens, status)), "gbs_kv_append")

    def read(self, seqs=None, cu_tokens=None, n_tokens: int | None = None, out=None, stream=None):
        """The rows that the cache stands for, [n_tokens, n_kv_heads, d] bf16 keys and values, in their own basis."""
        if out is None:
            if n_tokens is None:
                if cu_tokens is not None:
                    raise ValueError("gbs: n_tokens says how many rows cu_tokens (on the device) asks for")
                n_tokens = seqs.shape[0] if seqs is not None else self.page_table.shape[0]
            shape = (n_tokens, self.n_kv_heads, self.plan.info.d)
            out = tuple(self._empty(stream, shape, torch.bfloat16) for _ in range(2))
        k, v = out
        for what, x in (("k_out", k), ("v_out", v)):
            self._rows(what, x, self.n_kv_heads)
            _check_buffer(what, x, self.pages, torch.bfloat16, k.numel())
        s, cu, n = self._items(seqs, cu_tokens, k.shape[0])
        _check(lib().gbs_kv_read(self.plan.handle, ctypes.byref(self._c), s, cu, n, k.shape[0], k.data_ptr(), v.data_ptr(),
                                 self._stream(stream, k, v, seqs, cu_tokens)), "gbs_kv_read")
        return k, v

    def attention(self, q: torch.Tensor, seqs=None, cu_tokens=None, max_tokens: int | None = None, causal: bool = True, window: int = 0,
                  scale: float = 0.0, max_len: int = 0, out=None, stream=None) -> torch.Tensor:
        """Attention of query tokens q [tokens, heads, d] (bf16) over the cache; the same shape comes back.  max_tokens: no item has
        more tokens (None: as many as q has, or 1 without cu_tokens; it chooses the kernel and bounds what is looked through, so the closer
        the better, and items x max_tokens x heads / n_kv_heads may be 2^28 at most); max_len: about
        how long the longest sequence is (0: the table's width), by which the work is split; scale 0: 1 / sqrt(d).  Rows behind the last item's, and an item's beyond
        max_tokens, are left as they are in `out`, and undefined without one."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise ValueError("gbs: q must be [tokens, heads, d]")
        self._rows("q", q, q.shape[1])
        if max_tokens is None:
            max_tokens = max(1, q.shape[0]) if cu_tokens is not None else 1
        for what, v in (("max_tokens", max_tokens), ("window", window), ("max_len", max_len)):
            _int32(what, v)
        if out is None:
            out = self._empty(stream, q.shape, torch.bfloat16)
        self._rows("out", out, q.shape[1])
        if out.shape[0] != q.shape[0]:
            raise ValueError("gbs: q has %d tokens, out %d" % (q.shape[0], out.shape[0]))
        s, cu, n = self._items(seqs, cu_tokens, q.shape[0])
        need = ctypes.c_int64(0)
        _check(lib().gbs_kv_attention_workspace(self.plan.handle, ctypes.byref(self._c), q.shape[1], q.shape[0], max_tokens, ctypes.byref(need)),
               "gbs_kv_attention_workspace")
        work = self._empty(stream, need.value, torch.uint8, False)
        _check(lib().gbs_kv_attention(self.plan.handle, ctypes.byref(self._c), s, cu, n, q.shape[0], max_tokens, max_len, q.data_ptr(),
                                      *self._strides(q), q.shape[1], float(scale), window, GBS_KV_CAUSAL if causal else 0, out.data_ptr(),
                                      *self._strides(out), work.data_ptr(), need.value, self._stream(stream, q, out, seqs, cu_tokens)),
               "gbs_kv_attention")
        return out

    def shared_attention(self, q: torch.Tensor, seqs=None, cu_tokens=None, groups=None, max_tokens: int | None = None, causal: bool = True,
                         scale: float = 0.0, max_own: int = 0, max_prefix: int = 0, out=None, stream=None) -> torch.Tensor:
        """attention (without a window) for items whose sequences begin alike, as forks of one prompt do: the pages that all items of a group begin with are
        read once for the group.  groups: int32 [groups + 1], the first item of each group and the end (None: all items are one group); which pages
        are common is found in the page table.  max_own: about how many tokens the longest sequence has behind what its group shares; max_prefix: about how many the longest prefix has
        (0: the table's width, too much for a table with room to spare), by which the call judges whether sharing gains more than the 20 to 45 us that it costs; where that is not
        likely, it reads as attention does."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise ValueError("gbs: q must be [tokens, heads, d]")
        self._rows("q", q, q.shape[1])
        if max_tokens is None:
            max_tokens = max(1, q.shape[0]) if cu_tokens is not None else 1
        for what, v in (("max_tokens", max_tokens), ("max_own", max_own), ("max_prefix", max_prefix)):
            _int32(what, v)
        if out is None:
            out = self._empty(stream, q.shape, torch.bfloat16)
        self._rows("out", out, q.shape[1])
        if out.shape[0] != q.shape[0]:
            raise ValueError("gbs: q has %d tokens, out %d" % (q.shape[0], out.shape[0]))
        s, cu, n = self._items(seqs, cu_tokens, q.shape[0])
        if groups is not None and (not isinstance(groups, torch.Tensor) or groups.dim() != 1 or groups.shape[0] < 2):
            raise ValueError("gbs: groups must be one row of the groups' first items and the end")
        n_groups = groups.shape[0] - 1 if groups is not None else 1
        need = ctypes.c_int64(0)
        _check(lib().gbs_kv_shared_attention_workspace(self.plan.handle, ctypes.byref(self._c), n, q.shape[0], max_tokens, n_groups, max_prefix, q.shape[1],
                                                       ctypes.byref(need)), "gbs_kv_shared_attention_workspace")
        work = self._empty(stream, need.value, torch.uint8, False)
        _check(lib().gbs_kv_shared_attention(self.plan.handle, ctypes.byref(self._c), s, cu, n, q.shape[0], max_tokens,
                                             self._ints("groups", groups, n_groups + 1), n_groups, max_own, max_prefix, q.data_ptr(), *self._strides(q), q.shape[1],
                                             float(scale), GBS_KV_CAUSAL if causal else 0, out.data_ptr(), *self._strides(out), work.data_ptr(),
                                             need.value, self._stream(stream, q, out, seqs, cu_tokens, groups)), "gbs_kv_shared_attention")
        return out

    def _weights(self, what: str, t: torch.Tensor, width: int | None = None):
        """Weights of cached tokens: [sequences, n_kv_heads, width] fp32."""
        _check_buffer(what, t, self.pages, torch.float32, 1)
        if t.dim() != 3 or t.shape[0] != self.page_table.shape[0] or t.shape[1] != self.n_kv_heads or (width is not None and t.shape[2] != width):
            raise ValueError("gbs: %s must be [%d, %d, %s], got shape %s" % (what, self.page_table.shape[0], self.n_kv_heads,
                                                                            "width" if width is None else width, tuple(t.shape)))

    def attention_mass(self, q: torch.Tensor, mass: torch.Tensor, seqs=None, cu_tokens=None, max_tokens: int | None = None, decay: float = 1.0, base=None,
                       causal: bool = True, window: int = 0, scale: float = 0.0, stream=None) -> torch.Tensor:
        """The softmax weight that each cached token gets from query tokens q [tokens, heads, d] (bf16), summed over them and the query heads of a KV
        head, into mass [sequences, n_kv_heads, width] (fp32) at the token's position: mass = decay * base + the sum.  base: None is mass itself, what
        the calls before added up; the items' own tokens (the last ones of their sequences) start from 0, and with decay 0 all do.  Weights belong to positions: clear
        those of a sequence that begins anew, copy them for a fork.  Positions from width on are left out.  Returns mass."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise ValueError("gbs: q must be [tokens, heads, d]")
        self._rows("q", q, q.shape[1])
        if max_tokens is None:
            max_tokens = max(1, q.shape[0]) if cu_tokens is not None else 1
        for what, v in (("max_tokens", max_tokens), ("window", window)):
            _int32(what, v)
        self._weights("mass", mass)
        if base is None:
            base = mass
        self._weights("base", base, mass.shape[2])
        s, cu, n = self._items(seqs, cu_tokens, q.shape[0])
        need = ctypes.c_int64(0)
        _check(lib().gbs_kv_attention_mass_workspace(self.plan.handle, ctypes.byref(self._c), n, q.shape[0], max_tokens, q.shape[1], mass.shape[2],
                                                     ctypes.byref(need)), "gbs_kv_attention_mass_workspace")
        work = self._empty(stream, need.value, torch.uint8, False)
        _check(lib().gbs_kv_attention_mass(self.plan.handle, ctypes.byref(self._c), s, cu, n, q.shape[0], max_tokens, q.data_ptr(), *self._strides(q),
                                           q.shape[1], float(scale), window, GBS_KV_CAUSAL if causal else 0, base.data_ptr(), float(decay),
                                           mass.data_ptr(), mass.shape[2], work.data_ptr(), need.value,
                                           self._stream(stream, q, mass, base, seqs, cu_tokens)), "gbs_kv_attention_mass")
        return mass

    def evict(self, mass: torch.Tensor, keep: int, seqs=None, recent: int = 0, first: int = 0, into=None, stream=None):
        """Cut sequences longer than `keep` tokens down to `keep`, for each KV head its own: the first `first`, the last `recent`, and of those between the ones with
        the largest mass [sequences, n_kv_heads, width] (fp32, as attention_mass leaves it).  What stays moves to the front of the sequence, in order, into
        pages of its own (which have to be free), and its mass to the front of `into` (None: of mass).  Returns the items' status (GBS_KV_*) and the
        former positions of what stays [items, n_kv_heads, keep] (int32, -1 where there is none).  Behind what stays, `into` is as it was."""
        for what, v in (("keep", keep), ("recent", recent), ("first", first)):
            _int32(what, v)
        self._weights("mass", mass)
        if into is None:
            into = mass
        self._weights("into", into, mass.shape[2])
        n = seqs.shape[0] if seqs is not None else self.page_table.shape[0]
        status = self._empty(stream, n, torch.int32)
        kept = self._empty(stream, (n, self.n_kv_heads, max(keep, 0)), torch.int32)
        need = ctypes.c_int64(0)
        _check(lib().gbs_kv_evict_workspace(self.plan.handle, ctypes.byref(self._c), n, keep, ctypes.byref(need)), "gbs_kv_evict_workspace")
        work = self._empty(stream, need.value, torch.uint8, False)
        _check(lib().gbs_kv_evict(self.plan.handle, ctypes.byref(self._c), self._ints("seqs", seqs, n), n, keep, recent, first, mass.data_ptr(),
                                  into.data_ptr(), mass.shape[2], kept.data_ptr(), status.data_ptr(), work.data_ptr(), need.value,
                                  self._stream(stream, mass, into, seqs)), "gbs_kv_evict")
        return status, kept


# the methods that _native.so has a regular call for
_PYTHON_KV_METHODS = {name: KVCache.__dict__[name] for name in ("extend", "fork", "free", "compact", "append", "read", "attention", "shared_attention",
                                                                   "attention_mass", "evict")}
_PYTHON_METHODS = {name: Plan.__dict__[name] for name in ("rotate_quantize", "dequantize", "quantized_matmul", "clip_error")}


class HostPipeline:
    """Host-resident rows through one or more plans: pinned host -> device -> kernels -> pinned host.

    The rows are cut into `chunks` row ranges.  Chunk i+1 is copied to the device on a copy stream
    while chunk i is quantized and its codes and scales travel back on the compute stream, so the
    two PCIe directions work at the same time.  Only copies, events and the plans' launches happen
    here; staging buffers on the device are allocated once.
    """

    def __init__(self, plans, n_rows: int, device="cuda:0", chunks: int = 4, dtype=torch.bfloat16):
        self.plans = list(plans)
        d = self.plans[0].info.d
        assert all(p.info.d == d for p in self.plans)
        self.n_rows, self.d = n_rows, d
        chunks = max(1, min(chunks, n_rows)) if n_rows else 1
        step = (n_rows + chunks - 1) // chunks if n_rows else 0
        self.ranges = [(r, min(n_rows, r + step)) for r in range(0, n_rows, step)] if n_rows else []
        self.x_dev = torch.empty((n_rows, d), dtype=dtype, device=device)
        self.outs = [p.alloc_outputs(n_rows, device) for p in self.plans]
        self.copy_stream = torch.cuda.Stream(device=device)
        self.ev_in = [torch.cuda.Event() for _ in self.ranges]
        self.ev_start = torch.cuda.Event()
        # views of the staging buffers and the marshalled arguments of every launch, made once: the per-call host
        # work is what bounds a pipeline of short launches
        self.x_views = [self.x_dev[r0:r1] for r0, r1 in self.ranges]
        self.calls = []
        dt = _dtype_code(self.x_dev)
        for (r0, r1), xv in zip(self.ranges, self.x_views):
            per_plan = []
            for p, (codes, scales, _) in zip(self.plans, self.outs):
                cv, sv = codes[r0:r1], scales[r0:r1]
                per_plan.append((ctypes.c_void_p(p.handle), xv.data_ptr(), dt, r1 - r0, xv.stride(0) if r1 - r0 > 1 else d,
                                 cv.data_ptr(), sv.data_ptr(), cv, sv))
            self.calls.append(per_plan)

    def run(self, x_host: torch.Tensor, outs_host, stream=None):
        """outs_host: one (codes_host, scales_host) pair per plan.  Work is enqueued on `stream` (and the
        internal copy stream, joined to it); the caller synchronises `stream`."""
        s = stream or torch.cuda.current_stream()
        sp = int(s.cuda_stream)
        rq = lib().gbs_rotate_quantize
        self.ev_start.record(s)
        self.copy_stream.wait_event(self.ev_start)          # staging buffers of the previous call are free
        for i, (r0, r1) in enumerate(self.ranges):
            with torch.cuda.stream(self.copy_stream):
                self.x_views[i].copy_(x_host[r0:r1], non_blocking=True)
                self.ev_in[i].record(self.copy_stream)
            with torch.cuda.stream(s):
                s.wait_event(self.ev_in[i])
                for (h, xp, dt, n, stride, cp, scp, cv, sv), (ch, sh) in zip(self.calls[i], outs_host):
                    _check(rq(h, xp, dt, n, stride, cp, scp, None, sp), "gbs_rotate_quantize")
                    ch[r0:r1].copy_(cv, non_blocking=True)
                    sh[r0:r1].copy_(sv, non_blocking=True)
        return outs_host
