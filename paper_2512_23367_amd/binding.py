"""ctypes binding of libqlinear.so: same names as include/qlinear.h, argument marshalling only.

Tensors are torch CUDA (ROCm) tensors used as plain device buffers; every call is enqueued on
torch's current stream.  There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
import warnings
from importlib import import_module

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqlinear.so")

QL_OK = 0
STATUS_NAMES = {0: "QL_OK", 1: "QL_ERR_NULL", 2: "QL_ERR_SHAPE", 3: "QL_ERR_ALIGN",
                4: "QL_ERR_UNSUPPORTED", 5: "QL_ERR_WORKSPACE", 6: "QL_ERR_HIP"}

EXPORTS = [
    "ql_version", "ql_last_error", "ql_weight_bytes", "ql_act_kernel_bytes", "ql_workspace_bytes",
    "ql_quant_act_per_token", "ql_quant_act_rmsnorm", "ql_quant_act_swiglu", "ql_act_repack", "ql_quant_weight", "ql_export_canonical",
    "ql_w8a8_linear", "ql_w8a8_linear_static", "ql_w4a8_linear", "ql_w8a8_gemm", "ql_w4a8_gemm",
    "ql_w8a8_gemm_acc_i32", "ql_w4a8_gemm_acc_i32", "ql_set_kernel_variant", "ql_plan_gemm",
    "ql_hadamard_block", "ql_smooth_calibrate", "ql_smooth_scales",
    "ql_quant_act_per_token_transformed", "ql_quant_weight_transformed",
    "ql_act_scale_calibrate", "ql_quant_act_opt", "ql_quant_weight_opt",
    "ql_kv_cache_bytes", "ql_kv_resize", "ql_kv_append", "ql_kv_read", "ql_paged_attention_bytes", "ql_paged_attention",
]

QL_RANGE_SYMMETRIC, QL_RANGE_EQ2 = 0, 1
QL_FAMILY_DECODE, QL_FAMILY_TILE = 1, 2


class QlPlan(ctypes.Structure):
    """Mirror of the C struct ql_plan."""
    _fields_ = [("family", ctypes.c_int), ("variant", ctypes.c_int), ("tile_tokens", ctypes.c_int),
                ("tile_channels", ctypes.c_int), ("splits", ctypes.c_int), ("est_us", ctypes.c_double),
                ("rest_channels", ctypes.c_int), ("rest_variant", ctypes.c_int)]


class QlKvFormat(ctypes.Structure):
    """Mirror of the C struct ql_kv_format: QlKvFormat(heads=, head_dim=, page_size=, pages=, bits=)."""
    _fields_ = [("heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("page_size", ctypes.c_int), ("pages", ctypes.c_int),
                ("bits", ctypes.c_int)]


QL_SCOPE_FINE, QL_SCOPE_TENSOR, QL_SCOPE_STATIC = 0, 1, 2


class QlError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (python -m paper_2512_23367_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2512_23367_amd.build` "
                "(there is no CPU or PyTorch fallback)")
        l = ctypes.CDLL(LIB_PATH)
        c = ctypes
        vp, i, i64, sz = c.c_void_p, c.c_int, c.c_int64, c.c_size_t
        szp = c.POINTER(c.c_size_t)
        l.ql_version.restype = i
        l.ql_version.argtypes = []
        l.ql_last_error.restype = c.c_char_p
        l.ql_last_error.argtypes = []
        sigs = {
            "ql_set_kernel_variant": [i],
            "ql_plan_gemm": [i, i, i, i, i, sz, c.POINTER(QlPlan)],
            "ql_weight_bytes": [i, i, i, i, szp, szp, szp],
            "ql_act_kernel_bytes": [i, i, szp],
            "ql_workspace_bytes": [i, i, i, i, szp],
            "ql_quant_act_per_token": [vp, i64, i, i, vp, vp, vp, vp],
            "ql_quant_act_rmsnorm": [vp, i64, i, i, vp, c.c_float, vp, vp, vp, vp],
            "ql_quant_act_swiglu": [vp, i64, i, i, vp, vp, vp, vp],
            "ql_act_repack": [vp, i, i, vp, vp],
            "ql_quant_weight": [vp, i, i, i, i, vp, vp, vp, vp],
            "ql_export_canonical": [vp, i, i, i, i, vp, vp, vp],
            "ql_w8a8_linear": [vp, i64, i, i, vp, vp, vp, i, vp, i64, vp, sz, vp],
            "ql_w4a8_linear": [vp, i64, i, i, vp, i, vp, i, vp, i64, vp, sz, vp],
            "ql_w8a8_linear_static": [vp, i64, i, i, vp, vp, vp, i, vp, i64, vp],
            "ql_w8a8_gemm": [vp, vp, i, i, vp, vp, vp, i, vp, i64, vp, sz, vp],
            "ql_w4a8_gemm": [vp, vp, i, i, vp, i, vp, i, vp, i64, vp, sz, vp],
            "ql_w8a8_gemm_acc_i32": [vp, i, i, vp, i, vp, vp, sz, vp],
            "ql_w4a8_gemm_acc_i32": [vp, i, i, vp, i, i, vp, vp, i, i, vp, sz, vp],
            "ql_hadamard_block": [i, c.POINTER(c.c_int)],
            "ql_smooth_calibrate": [vp, i64, i, i, vp, vp],
            "ql_smooth_scales": [vp, vp, i, i, c.c_float, vp, vp, vp],
            "ql_quant_act_per_token_transformed": [vp, i64, i, i, vp, i, vp, vp, vp, vp],
            "ql_quant_weight_transformed": [vp, i, i, i, i, vp, i, vp, vp, vp, vp, vp],
            "ql_act_scale_calibrate": [vp, i64, i, i, i, vp, vp],
            "ql_quant_act_opt": [vp, i64, i, i, i, i, vp, vp, vp, vp, vp, vp],
            "ql_quant_weight_opt": [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp],
            "ql_kv_cache_bytes": [c.POINTER(QlKvFormat), szp],
            "ql_kv_resize": [vp, vp, i, i, vp, i, vp, vp, vp, i64, i, vp, vp, vp, vp, i, vp],
            "ql_kv_append": [vp, i64, vp, i64, vp, i64, i, i, vp, i, i, vp, vp, vp, i64, vp, c.POINTER(QlKvFormat), vp],
            "ql_kv_read": [vp, c.POINTER(QlKvFormat), vp, i, vp, i64, vp, i64, vp],
            "ql_paged_attention_bytes": [c.POINTER(QlKvFormat), i, i, i, i, szp],
            "ql_paged_attention": [vp, i64, i, i, vp, c.POINTER(QlKvFormat), vp, i64, i, vp, vp, vp, i, c.c_float, i, i, i, vp, i64, vp, sz, vp],
        }
        for name, args in sigs.items():
            fn = getattr(l, name)
            fn.restype = i
            fn.argtypes = args
        _lib = l
        _bind_native(l)
    return _lib


# Native argument marshalling (csrc/pycall.cpp) of the calls that are made per layer: the checks below in C++, then the library, or
# None for anything unusual, which then takes the Python below.  None before the library is loaded, or without the module.
_native = None


def _bind_native(l):
    global _native
    try:
        _qlcall = import_module(f"{__package__}._qlcall")
    except ModuleNotFoundError:
        return
    except ImportError as e:
        warnings.warn(f"the call module _qlcall does not load, calls are marshalled in Python, 2 to 3 us slower each (built against another "
                      f"torch? rebuild with `python -m paper_2512_23367_amd.build`): {e}", RuntimeWarning)
        return
    names = ("ql_weight_bytes", "ql_act_kernel_bytes", "ql_w8a8_linear", "ql_w4a8_linear", "ql_w8a8_gemm", "ql_w4a8_gemm",
             "ql_quant_act_per_token", "ql_quant_act_rmsnorm", "ql_quant_act_swiglu", "ql_quant_act_per_token_transformed")
    cache_names = ("ql_kv_cache_bytes", "ql_kv_resize", "ql_kv_append", "ql_kv_read", "ql_paged_attention")
    addresses = lambda names: tuple(ctypes.cast(getattr(l, n), ctypes.c_void_p).value for n in names)  # noqa: E731
    _qlcall.bind(addresses(names))
    _qlcall.bind_cache(addresses(cache_names))
    _qlcall.bind_format(QlKvFormat)
    _native = _qlcall


def _done(status) -> bool:
    """Whether the native call was made (raises if the library refused it)."""
    if status is None:
        return False
    _check(status)
    return True


def _check(status: int):
    if status != QL_OK:
        raise QlError(status, lib().ql_last_error().decode())


def _p(t):
    """Device pointer of a tensor (None -> NULL), as the integer that a pointer argument takes."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    return t.data_ptr()


# Handle of torch's current stream.  torch.cuda.current_stream() builds a Stream object first: 2.7 us of a call that the
# library itself takes 3.7 us for (one token through 1536 x 1536), against 0.1 us here.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _current_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _want(t, dtype, name):
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return t


def ql_version() -> int:
    return lib().ql_version()


def ql_last_error() -> str:
    return lib().ql_last_error().decode()


def ql_set_kernel_variant(variant: int):
    _check(lib().ql_set_kernel_variant(variant))


def ql_plan_gemm(M: int, N: int, K: int, bits: int, group: int, scratch_bytes: int = 0) -> QlPlan:
    """What the automatic choice launches for this GEMM shape and the estimate it goes by (host only)."""
    plan = QlPlan()
    _check(lib().ql_plan_gemm(M, N, K, bits, group, scratch_bytes, ctypes.byref(plan)))
    return plan


def ql_hadamard_block(K: int) -> int:
    b = ctypes.c_int()
    _check(lib().ql_hadamard_block(K, ctypes.byref(b)))
    return b.value


def ql_smooth_calibrate(x, xmax):
    _want(x, torch.float16, "x"), _want(xmax, torch.float32, "xmax")
    M, K = x.shape
    _check(lib().ql_smooth_calibrate(_p(x), _ld(x) if M else K, M, K, _p(xmax), _stream()))


def ql_smooth_scales(xmax, w, alpha, smooth, inv_smooth):
    _want(w, torch.float16, "w"), _want(xmax, torch.float32, "xmax")
    N, K = w.shape
    _check(lib().ql_smooth_scales(_p(xmax), _p(w), N, K, float(alpha), _p(smooth), _p(inv_smooth), _stream()))


def ql_quant_act_per_token_transformed(x, inv_smooth, hadamard_block, xq_rowmajor, xq_kernel, sx):
    if _native is not None and _done(_native.quant_transformed(x, inv_smooth, hadamard_block, xq_rowmajor, xq_kernel, sx, _stream)):
        return
    _want(x, torch.float16, "x")
    M, K = x.shape
    _check(lib().ql_quant_act_per_token_transformed(_p(x), _ld(x) if M else K, M, K, _p(inv_smooth), hadamard_block,
                                                    _p(xq_rowmajor), _p(xq_kernel), _p(sx), _stream()))


def ql_quant_weight_transformed(w, bits, group, smooth, hadamard_block, w32, wq_canonical, scales, wq_kernel):
    _want(w, torch.float16, "w"), _want(w32, torch.float32, "w32")
    N, K = w.shape
    _check(lib().ql_quant_weight_transformed(_p(w), N, K, bits, group, _p(smooth), hadamard_block, _p(w32),
                                             _p(wq_canonical), _p(scales), _p(wq_kernel), _stream()))


def ql_act_scale_calibrate(x, rng, scale):
    _want(x, torch.float16, "x"), _want(scale, torch.float32, "scale")
    M, K = x.shape
    _check(lib().ql_act_scale_calibrate(_p(x), _ld(x) if M else K, M, K, rng, _p(scale), _stream()))


def ql_quant_act_opt(x, rng, scope, static_scale, xq_rowmajor, xq_kernel, sx, scratch):
    _want(x, torch.float16, "x")
    M, K = x.shape
    _check(lib().ql_quant_act_opt(_p(x), _ld(x) if M else K, M, K, rng, scope, _p(static_scale), _p(xq_rowmajor),
                                  _p(xq_kernel), _p(sx), _p(scratch), _stream()))


def ql_quant_weight_opt(w, bits, group, rng, scope, wq_canonical, scales, wq_kernel, scratch):
    _want(w, torch.float16, "w")
    N, K = w.shape
    _check(lib().ql_quant_weight_opt(_p(w), N, K, bits, group, rng, scope, _p(wq_canonical), _p(scales),
                                     _p(wq_kernel), _p(scratch), _stream()))


def ql_weight_bytes(N, K, bits, group):
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().ql_weight_bytes(N, K, bits, group, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


# The checks of every GEMM call ask for these two: functions of the sizes alone, kept by value.  (64.0 finds the size of 64
# here and is refused by the call itself; kept per type as well the smallest call took 1 % longer.)
@functools.lru_cache(maxsize=4096)
def _blob_bytes(N, K, bits, group) -> int:
    return ql_weight_bytes(N, K, bits, group)[2]


@functools.lru_cache(maxsize=4096)
def _act_bytes(M, K) -> int:
    return ql_act_kernel_bytes(M, K)


def ql_act_kernel_bytes(M, K) -> int:
    a = ctypes.c_size_t()
    _check(lib().ql_act_kernel_bytes(M, K, ctypes.byref(a)))
    return a.value


def ql_workspace_bytes(M, N, K, bits) -> int:
    a = ctypes.c_size_t()
    _check(lib().ql_workspace_bytes(M, N, K, bits, ctypes.byref(a)))
    return a.value


def _ld(t):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("2-D tensor with unit inner stride expected")
    return t.stride(0)


def ql_quant_act_per_token(x, xq_rowmajor=None, xq_kernel=None, sx=None):
    if _native is not None and _done(_native.quant_act(x, xq_rowmajor, xq_kernel, sx, _stream)):
        return
    _want(x, torch.float16, "x")
    M, K = x.shape
    _check(lib().ql_quant_act_per_token(_p(x), _ld(x) if M else K, M, K, _p(xq_rowmajor), _p(xq_kernel), _p(sx),
                                        _stream()))


def ql_quant_act_rmsnorm(x, gamma, eps, xq_rowmajor=None, xq_kernel=None, sx=None):
    if _native is not None and _done(_native.quant_rmsnorm(x, gamma, eps, xq_rowmajor, xq_kernel, sx, _stream)):
        return
    _want(x, torch.float16, "x"), _want(gamma, torch.float16, "gamma")
    M, K = x.shape
    _check(lib().ql_quant_act_rmsnorm(_p(x), _ld(x) if M else K, M, K, _p(gamma), float(eps), _p(xq_rowmajor),
                                      _p(xq_kernel), _p(sx), _stream()))


def ql_quant_act_swiglu(gate_up, xq_rowmajor=None, xq_kernel=None, sx=None):
    """gate_up: fp16 [M, 2F] (gate half, then up half); quantizes silu(gate) * up per token (K = F)."""
    if _native is not None and _done(_native.quant_swiglu(gate_up, xq_rowmajor, xq_kernel, sx, _stream)):
        return
    _want(gate_up, torch.float16, "gate_up")
    M, F2 = gate_up.shape
    if F2 % 2:
        raise ValueError("gate_up has an even number of columns")
    _check(lib().ql_quant_act_swiglu(_p(gate_up), _ld(gate_up) if M else F2, M, F2 // 2, _p(xq_rowmajor), _p(xq_kernel),
                                     _p(sx), _stream()))


def ql_act_repack(xq_rowmajor, xq_kernel):
    _want(xq_rowmajor, torch.int8, "xq_rowmajor")
    M, K = xq_rowmajor.shape
    _check(lib().ql_act_repack(_p(xq_rowmajor), M, K, _p(xq_kernel), _stream()))


def ql_quant_weight(w, bits, group, wq_canonical=None, scales=None, wq_kernel=None):
    _want(w, torch.float16, "w")
    N, K = w.shape
    if not w.is_contiguous():
        raise ValueError("w must be contiguous")
    _check(lib().ql_quant_weight(_p(w), N, K, bits, group, _p(wq_canonical), _p(scales), _p(wq_kernel), _stream()))


def ql_export_canonical(wq_kernel, N, K, bits, group, wq_canonical=None, scales=None):
    _check(lib().ql_export_canonical(_p(wq_kernel), N, K, bits, group, _p(wq_canonical), _p(scales), _stream()))


def _ws(ws):
    return (_p(ws), ws.nbytes) if ws is not None else (None, 0)


def _nbytes(t):
    return t.nbytes


def _check_gemm_buffers(M, K, N, bits, group, w_kernel, sw, bias, y, xq_kernel=None, sx=None):
    """Host-side size checks the C side cannot make (it sees pointers only): a buffer that is too small or of the
    wrong layout would be read or written out of bounds by the kernels."""
    if w_kernel is None or w_kernel.nbytes < _blob_bytes(N, K, bits, group):
        raise ValueError("w_kernel is smaller than the kernel-layout blob of ql_weight_bytes (canonical codes passed?)")
    if y.shape != (M, N) or (M and y.stride(1) != 1):
        raise ValueError(f"y must be [M,N] = [{M},{N}] with unit inner stride")
    if bits == 8 and (sw is None or sw.numel() < N):
        raise ValueError("sw needs N fp32 entries")
    if bias is not None and (bias.dtype != torch.float16 or bias.numel() < N):
        raise ValueError("bias must be fp16 with N entries")
    if xq_kernel is not None and _nbytes(xq_kernel) < _act_bytes(M, K):
        raise ValueError("xq_kernel is smaller than ql_act_kernel_bytes")
    if sx is not None and (sx.dtype != torch.float32 or sx.numel() < M):
        raise ValueError("sx needs M fp32 entries")


def ql_w8a8_linear(x, wq_kernel, sw, bias, N, y, ws):
    if _native is not None and _done(_native.w8a8_linear(x, wq_kernel, sw, bias, N, y, ws, _stream)):
        return
    _want(x, torch.float16, "x"), _want(y, torch.float16, "y"), _want(sw, torch.float32, "sw")
    M, K = x.shape
    _check_gemm_buffers(M, K, N, 8, 0, wq_kernel, sw, bias, y)
    wsp, wsb = _ws(ws)
    _check(lib().ql_w8a8_linear(_p(x), _ld(x) if M else K, M, K, _p(wq_kernel), _p(sw), _p(bias), N, _p(y),
                                _ld(y) if M else N, wsp, wsb, _stream()))


def ql_w8a8_linear_static(x, wq_kernel, sw, bias, N, y):
    """ql_w8a8_linear on the library's own static workspace (allocates nothing)."""
    _want(x, torch.float16, "x"), _want(y, torch.float16, "y"), _want(sw, torch.float32, "sw")
    M, K = x.shape
    _check_gemm_buffers(M, K, N, 8, 0, wq_kernel, sw, bias, y)
    _check(lib().ql_w8a8_linear_static(_p(x), _ld(x) if M else K, M, K, _p(wq_kernel), _p(sw), _p(bias), N, _p(y),
                                       _ld(y) if M else N, _stream()))


def ql_w4a8_linear(x, w4_kernel, group, bias, N, y, ws):
    if _native is not None and _done(_native.w4a8_linear(x, w4_kernel, group, bias, N, y, ws, _stream)):
        return
    _want(x, torch.float16, "x"), _want(y, torch.float16, "y")
    M, K = x.shape
    _check_gemm_buffers(M, K, N, 4, group, w4_kernel, None, bias, y)
    wsp, wsb = _ws(ws)
    _check(lib().ql_w4a8_linear(_p(x), _ld(x) if M else K, M, K, _p(w4_kernel), group, _p(bias), N, _p(y),
                                _ld(y) if M else N, wsp, wsb, _stream()))


def ql_w8a8_gemm(xq_kernel, sx, M, K, wq_kernel, sw, bias, N, y, ws=None):
    if _native is not None and _done(_native.w8a8_gemm(xq_kernel, sx, M, K, wq_kernel, sw, bias, N, y, ws, _stream)):
        return
    _want(y, torch.float16, "y")
    _check_gemm_buffers(M, K, N, 8, 0, wq_kernel, sw, bias, y, xq_kernel, sx)
    wsp, wsb = _ws(ws)
    _check(lib().ql_w8a8_gemm(_p(xq_kernel), _p(sx), M, K, _p(wq_kernel), _p(sw), _p(bias), N, _p(y),
                              _ld(y) if M else N, wsp, wsb, _stream()))


def ql_w4a8_gemm(xq_kernel, sx, M, K, w4_kernel, group, bias, N, y, ws=None):
    if _native is not None and _done(_native.w4a8_gemm(xq_kernel, sx, M, K, w4_kernel, group, bias, N, y, ws, _stream)):
        return
    _want(y, torch.float16, "y")
    _check_gemm_buffers(M, K, N, 4, group, w4_kernel, None, bias, y, xq_kernel, sx)
    wsp, wsb = _ws(ws)
    _check(lib().ql_w4a8_gemm(_p(xq_kernel), _p(sx), M, K, _p(w4_kernel), group, _p(bias), N, _p(y),
                              _ld(y) if M else N, wsp, wsb, _stream()))


def ql_w8a8_gemm_acc_i32(xq_kernel, M, K, wq_kernel, N, acc, ws=None):
    _want(acc, torch.int32, "acc")
    if acc.numel() < M * N or not acc.is_contiguous():
        raise ValueError("acc must be a contiguous int32 [M,N]")
    if _nbytes(wq_kernel) < ql_weight_bytes(N, K, 8, 0)[2] or _nbytes(xq_kernel) < ql_act_kernel_bytes(M, K):
        raise ValueError("wq_kernel / xq_kernel smaller than their size queries report")
    wsp, wsb = _ws(ws)
    _check(lib().ql_w8a8_gemm_acc_i32(_p(xq_kernel), M, K, _p(wq_kernel), N, _p(acc), wsp, wsb, _stream()))


def ql_w4a8_gemm_acc_i32(xq_kernel, M, K, w4_kernel, group, N, acc, partials=None, row0=0, nrows=0, ws=None):
    _want(acc, torch.int32, "acc")
    if acc.numel() < M * N or not acc.is_contiguous():
        raise ValueError("acc must be a contiguous int32 [M,N]")
    if _nbytes(w4_kernel) < ql_weight_bytes(N, K, 4, group)[2] or _nbytes(xq_kernel) < ql_act_kernel_bytes(M, K):
        raise ValueError("w4_kernel / xq_kernel smaller than their size queries report")
    if partials is not None and (partials.dtype != torch.int32 or partials.numel() < nrows * (K // group) * N):
        raise ValueError("partials must be int32 [nrows, K/group, N]")
    wsp, wsb = _ws(ws)
    _check(lib().ql_w4a8_gemm_acc_i32(_p(xq_kernel), M, K, _p(w4_kernel), group, N, _p(acc), _p(partials), row0,
                                      nrows, wsp, wsb, _stream()))


# ---- the paged key/value cache and attention over it ----

def _here(*tensors):
    """All on the device whose stream the call goes to."""
    at = torch.cuda.current_device() if _current_device is None else _current_device()
    for t in tensors:
        if t is not None and (not t.is_cuda or t.get_device() != at):
            raise ValueError("tensors of the current device expected")


def _ints(t, name, n):
    _want(t, torch.int32, name)
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with at least {n} entries")
    return t.data_ptr()


def _heads_of(t, name, rows, head_dim):
    """Heads in the columns of fp16 [rows, heads * head_dim] with unit inner stride."""
    _want(t, torch.float16, name)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] % head_dim or (t.numel() and t.stride(1) != 1):
        raise ValueError(f"{name} must be [{rows}, heads * {head_dim}] with unit inner stride")
    return t.shape[1] // head_dim


def _row_stride(t):
    """The leading dimension of a checked matrix (torch gives a single row any stride: its columns, rounded up, do as well)."""
    return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + 7) // 8 * 8


def _kv_rows(t, name, rows, fmt):
    if _heads_of(t, name, rows, fmt.head_dim) != fmt.heads:
        raise ValueError(f"{name} must have the cache's {fmt.heads} heads of {fmt.head_dim}")


@functools.lru_cache(maxsize=256)
def _cache_bytes(*sizes) -> int:
    a = ctypes.c_size_t()
    _check(lib().ql_kv_cache_bytes(ctypes.byref(QlKvFormat(*sizes)), ctypes.byref(a)))
    return a.value


def ql_kv_cache_bytes(fmt: QlKvFormat) -> int:
    return _cache_bytes(fmt.heads, fmt.head_dim, fmt.page_size, fmt.pages, fmt.bits)


def _cache(cache, fmt):
    if not cache.is_contiguous() or cache.nbytes < ql_kv_cache_bytes(fmt):
        raise ValueError("cache must be contiguous with at least the bytes of ql_kv_cache_bytes")
    return cache.data_ptr()


def _table(t, requests):
    _want(t, torch.int32, "block_table")
    if t.dim() != 2 or t.shape[0] < requests or (t.numel() and t.stride(1) != 1):
        raise ValueError(f"block_table must be [{requests}, columns] with unit inner stride")
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else t.shape[1]), t.shape[1]


def ql_kv_resize(page_size, old_len, want_len, ring, pool, pool_out, block_table, kv_len, cu_new, slots, positions):
    """Pages, slots and positions for requests that go from old_len to want_len tokens; all int32 tensors on the device.
    The pool has ring.numel() pages; slots and positions have room for the step's new tokens."""
    if _native is not None and _done(_native.kv_resize(page_size, old_len, want_len, ring, pool, pool_out, block_table, kv_len, cu_new, slots, positions, _stream)):
        return
    _here(old_len, want_len, ring, pool, pool_out, block_table, kv_len, cu_new, slots, positions)
    n, most = old_len.numel(), min(slots.numel(), positions.numel())
    table, ld, columns = _table(block_table, n)
    _check(lib().ql_kv_resize(_ints(old_len, "old_len", n), _ints(want_len, "want_len", n), n, page_size, _ints(ring, "ring", 1), ring.numel(),
                              _ints(pool, "pool", 4), _ints(pool_out, "pool_out", 4), table, ld, columns, _ints(kv_len, "kv_len", n),
                              _ints(cu_new, "cu_new", n + 1), _ints(slots, "slots", most), _ints(positions, "positions", most), most, _stream()))


def ql_kv_append(q, k, v, cos_sin, positions, slots, q_out, cache, fmt):
    """Rotates q (into q_out, which may be q) and k by cos_sin (fp32 [positions, rotary_dim], or None) and stores k and v."""
    if _native is not None and _done(_native.kv_append(q, k, v, cos_sin, positions, slots, q_out, cache, fmt, _stream)):
        return
    _here(q, k, v, cos_sin, positions, slots, q_out, cache)
    T = k.shape[0]
    _kv_rows(k, "k", T, fmt), _kv_rows(v, "v", T, fmt)
    q_heads = rotary = most = 0
    if cos_sin is not None:
        _want(cos_sin, torch.float32, "cos_sin")
        if cos_sin.dim() != 2 or not cos_sin.is_contiguous():
            raise ValueError("cos_sin must be a contiguous [positions, rotary_dim]")
        most, rotary = cos_sin.shape
        _ints(positions, "positions", T)
    if q is not None:
        q_heads = _heads_of(q, "q", T, fmt.head_dim)
        if q_out is None or q_out.shape != q.shape or _heads_of(q_out, "q_out", T, fmt.head_dim) != q_heads:
            raise ValueError("q_out must have q's shape")
        if T == 0:                                        # (no rows have no address, which would mean no q)
            q, q_out, q_heads = None, None, 0
    _check(lib().ql_kv_append(_p(q), _row_stride(q) if q is not None else 0, k.data_ptr(), _row_stride(k), v.data_ptr(), _row_stride(v), T, q_heads,
                              _p(cos_sin), rotary, most, _p(positions), _ints(slots, "slots", T), _p(q_out),
                              _row_stride(q_out) if q_out is not None else 0, _cache(cache, fmt), ctypes.byref(fmt), _stream()))


def ql_kv_read(cache, fmt, slots, k=None, v=None):
    """Keys and values of the given slots as fp16 [T, heads * head_dim] (either may be None)."""
    if _native is not None and _done(_native.kv_read(cache, fmt, slots, k, v, _stream)):
        return
    _here(cache, slots, k, v)
    T = (k if k is not None else v if v is not None else slots).shape[0]
    for t, name in ((k, "k"), (v, "v")):
        if t is not None:
            _kv_rows(t, name, T, fmt)
    _check(lib().ql_kv_read(_cache(cache, fmt), ctypes.byref(fmt), _ints(slots, "slots", T), T, _p(k), _row_stride(k) if k is not None else 0,
                            _p(v), _row_stride(v) if v is not None else 0, _stream()))


def ql_paged_attention_bytes(fmt: QlKvFormat, T: int, requests: int, q_heads: int, max_new: int = 0) -> int:
    a = ctypes.c_size_t()
    _check(lib().ql_paged_attention_bytes(ctypes.byref(fmt), T, requests, q_heads, max_new, ctypes.byref(a)))
    return a.value


def ql_paged_attention(q, cache, fmt, block_table, cu_new, ctx_len, kv_len, scale, y, ws=None, causal=True, window=0, max_new=0):
    """Attention of the new tokens q (rows cu_new[b] .. of request b) over the cache; ws: ql_paged_attention_bytes of the same sizes."""
    if _native is not None and _done(_native.paged_attention(q, cache, fmt, block_table, cu_new, ctx_len, kv_len, scale, y, ws, causal, window, max_new, _stream)):
        return
    _here(q, cache, block_table, cu_new, ctx_len, kv_len, y, ws)
    T, n = q.shape[0], kv_len.numel()
    q_heads = _heads_of(q, "q", T, fmt.head_dim)
    if y.shape != q.shape or _heads_of(y, "y", T, fmt.head_dim) != q_heads:
        raise ValueError("y must have q's shape")
    if ctx_len is not None:
        _ints(ctx_len, "ctx_len", n)
    table, ld, columns = _table(block_table, n)
    wsp, wsb = _ws(ws)
    _check(lib().ql_paged_attention(q.data_ptr(), _row_stride(q), T, q_heads, _cache(cache, fmt), ctypes.byref(fmt), table, ld, columns,
                                    _ints(cu_new, "cu_new", n + 1), _p(ctx_len), _ints(kv_len, "kv_len", n), n, float(scale), int(causal), window,
                                    max_new, y.data_ptr(), _row_stride(y), wsp, wsb, _stream()))
