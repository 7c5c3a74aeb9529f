"""Thin ctypes binding of libpifa (include/pifa.h).

Argument marshalling only: every function has the name of the C entry point
it calls, takes torch tensors for device buffers (or numpy arrays for host
index arrays) and raises :class:`PifaError` on a non-OK status.  All compute
runs in the HIP library; if it is missing, loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
import threading

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpifa.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "pifa.h")

PIFA_F32 = 0
PIFA_BF16 = 1

PIFA_OK = 0
PIFA_ERR_INVALID_ARG = -1
PIFA_ERR_BAD_INDEX = -2
PIFA_ERR_UNSUPPORTED = -3
PIFA_ERR_HIP = -4
PIFA_ERR_OOM = -5
PIFA_ERR_NOT_RANK_R = -6
PIFA_ERR_NOT_SPD = -7
PIFA_ERR_WRONG_DEVICE = -8
PIFA_ERR_TOO_LARGE = -9


class pifa_dims(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("r", ctypes.c_int64)]


class adamw_tensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("p_bf16", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double)]


class PifaError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: %s" % (fn, pifa_status_string(status)))


_lock = threading.Lock()
_lib = None

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_i32p = ctypes.POINTER(ctypes.c_int32)
_f32 = ctypes.c_float
_f64 = ctypes.c_double
_st = ctypes.c_int

_SIGNATURES = {
    "pifa_status_string": (ctypes.c_char_p, [_st]),
    "pifa_validate_partition": (_st, [_i32p, _i32p, pifa_dims]),
    "pifa_gemm_plan": (_st, [_i64, _i64, _i64, ctypes.c_int, ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                             ctypes.POINTER(_i64)]),
    "pifa_layer_create": (_st, [_vp, _vp, _i32p, _i32p, pifa_dims, ctypes.c_int, ctypes.POINTER(_vp)]),
    "pifa_layer_destroy": (_st, [_vp]),
    "pifa_layer_reserve": (_st, [_vp, _i64]),
    "pifa_forward": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "pifa_forward_noalloc": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "pifa_layer_weight_bytes": (ctypes.c_size_t, [_vp]),
    "pifa_layer_set_intermediate_scale": (_st, [_vp, ctypes.c_int]),
    "pifa_layer_overflow_count": (_st, [_vp, ctypes.POINTER(_i64)]),
    "dense_forward": (_st, [_vp, _vp, _vp, _i64, _i64, _i64, ctypes.c_int, _vp]),
    "dense_layer_create": (_st, [_vp, _i64, _i64, ctypes.c_int, ctypes.POINTER(_vp)]),
    "dense_layer_forward": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "dense_layer_destroy": (_st, [_vp]),
    "dense_layer_reserve": (_st, [_vp, _i64]),
    "lowrank_uv_forward": (_st, [_vp, _vp, _vp, _vp, _i64, pifa_dims, ctypes.c_int, _vp]),
    "lowrank_layer_create": (_st, [_vp, _vp, pifa_dims, ctypes.c_int, ctypes.POINTER(_vp)]),
    "lowrank_layer_forward": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "lowrank_layer_reserve": (_st, [_vp, _i64]),
    "lowrank_layer_destroy": (_st, [_vp]),
    "pifa_layer_backward": (_st, [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp]),
    "pifa_group_create": (_st, [ctypes.c_int, ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_i32p),
                                ctypes.POINTER(_i32p), ctypes.POINTER(pifa_dims), ctypes.c_int,
                                ctypes.POINTER(_vp)]),
    "pifa_group_destroy": (_st, [_vp]),
    "pifa_group_reserve": (_st, [_vp, _i64]),
    "pifa_group_forward": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "pifa_group_weight_bytes": (ctypes.c_size_t, [_vp]),
    "pifa_group_set_intermediate_scale": (_st, [_vp, ctypes.c_int]),
    "pifa_group_overflow_count": (_st, [_vp, ctypes.POINTER(_i64)]),
    "pifa_calib_create": (_st, [_i64, ctypes.POINTER(_vp)]),
    "pifa_calib_destroy": (_st, [_vp]),
    "pifa_calib_reset": (_st, [_vp, _vp]),
    "pifa_calib_accumulate": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "pifa_calib_read": (_st, [_vp, _vp, _vp, _vp]),
    "pifa_calib_reconstruct": (_st, [_vp, _vp, _i64, _vp, _i64, ctypes.c_double, ctypes.c_double, _vp, _vp, _vp]),
    "pifa_build_f64": (_st, [_vp, pifa_dims, _vp, _vp, _i32p, _i32p, ctypes.POINTER(ctypes.c_double), _vp]),
    "rms_norm_forward": (_st, [_vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, ctypes.c_int, _vp]),
    "rms_norm_forward_e4m3": (_st, [_vp, _vp, _vp, _f32, _vp, _vp, _vp, _i64, _i64, ctypes.c_int, _vp]),
    "rms_norm_backward": (_st, [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, ctypes.c_int, _vp, ctypes.c_size_t,
                                _vp]),
    "rms_norm_backward_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "q4_layer_create": (_st, [_vp, _i64, _i64, ctypes.c_int, ctypes.POINTER(_vp)]),
    "q4_layer_create_mx": (_st, [_vp, _vp, _i64, _i64, ctypes.POINTER(_vp)]),
    "q4_layer_destroy": (_st, [_vp]),
    "q4_layer_read": (_st, [_vp, _vp, _vp, _vp]),
    "q4_layer_weight_bytes": (ctypes.c_size_t, [_vp]),
    "q4_layer_forward": (_st, [_vp, _vp, _vp, _i64, _vp]),
    "q4_layer_forward_e4m3": (_st, [_vp, _vp, _vp, _vp, _i64, _vp]),
    "q4_layer_norm_forward": (_st, [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _vp]),
    "q4_layer_reserve": (_st, [_vp, _i64]),
    "layer_norm_forward": (_st, [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, ctypes.c_int, _vp]),
    "layer_norm_backward": (_st, [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _i64, _i64, ctypes.c_int, _vp,
                                  ctypes.c_size_t, _vp]),
    "layer_norm_backward_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "adapter_plan": (_st, [_vp, _i64, _i64, _vp, ctypes.c_size_t, _vp]),
    "adapter_plan_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "adapter_forward": (_st, [_vp] * 7 + [_i64] * 5 + [_vp, ctypes.c_size_t, _vp]),
    "adapter_forward_bytes": (ctypes.c_size_t, [_i64] * 5),
    "adapter_backward": (_st, [_vp] * 10 + [_i64] * 5 + [_vp, ctypes.c_size_t, _vp]),
    "adapter_backward_bytes": (ctypes.c_size_t, [_i64] * 5),
    "adamw_create": (_st, [ctypes.POINTER(adamw_tensor), _i64, ctypes.c_int, ctypes.c_int, ctypes.c_uint32,
                           ctypes.POINTER(_vp)]),
    "adamw_destroy": (_st, [_vp]),
    "adamw_step": (_st, [_vp, _f64, _f64, _f64, _f64, _i64, _vp, _vp]),
    "adamw_count": (_st, [_vp, ctypes.POINTER(_i64)]),
    "pifa_probe_mfma": (_st, [_i64, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]),
    "pifa_probe_mfma_random": (_st, [_i64, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]),
    "pifa_probe_hbm_read": (_st, [_vp, _i64, ctypes.c_int, ctypes.POINTER(ctypes.c_double), _vp]),
    "pifa_profile_enable": (_st, [ctypes.c_int]),
    "pifa_profile_reset": (_st, []),
    "pifa_profile_read": (_st, [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(_i64),
                                ctypes.POINTER(ctypes.c_double), ctypes.c_int, ctypes.POINTER(ctypes.c_int)]),
}


def lib():
    """Open libpifa.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:  # set once, when it is ready
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError("libpifa.so not built: run `python -m paper_2501_19090_amd.build`")
            handle = ctypes.CDLL(LIB_PATH)
            for name, (res, args) in _SIGNATURES.items():
                fn = getattr(handle, name)
                fn.restype = res
                fn.argtypes = args
            _lib = handle
        return _lib


def declared_symbols(header: str = HEADER_PATH):
    """Function names declared in include/pifa.h."""
    with open(header) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b([a-z_][a-z0-9_]*)\s*\(", text)) - {"defined"})


# ---------------------------------------------------------------- marshalling
def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return PIFA_BF16
    if t.dtype == torch.float32:
        return PIFA_F32
    raise TypeError("unsupported dtype %s (bf16 or fp32)" % t.dtype)


def _dev_ptr(t, name: str) -> int | None:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


# Dimensions of the live handles created through this module.  The library
# takes raw pointers and cannot see how large a tensor is, so the calls below
# check that each buffer holds the bytes the call will read or write (a short
# buffer would be accessed past its end on the GPU).  Handles created
# elsewhere are passed through unchecked.
_dims: dict = {}
_dims_lock = threading.Lock()


def _esize(dt: int) -> int:
    return 2 if dt == PIFA_BF16 else 4


def _need(t, nbytes: int, name: str) -> None:
    if t is not None and t.numel() * t.element_size() < nbytes:
        raise ValueError("%s holds %d bytes, the call needs %d" % (name, t.numel() * t.element_size(), nbytes))


def _torch_dtype(dt: int):
    import torch
    return {PIFA_BF16: torch.bfloat16, PIFA_F32: torch.float32}.get(dt, torch.float64 if dt == "f64" else None)


def _same(t, name: str, dt, device=None) -> None:
    """t (if given) has element type dt (PIFA_BF16, PIFA_F32 or "f64") and lives
    on the given device index: the library reads raw bytes, so a tensor of
    another type or on another GPU would be misread, not rejected."""
    if t is None:
        return
    want = _torch_dtype(dt)
    if want is not None and t.dtype != want:
        raise TypeError("%s is %s, the call expects %s" % (name, t.dtype, want))
    if device is not None and t.is_cuda and t.device.index != device:
        raise ValueError("%s is on cuda:%d, the handle on cuda:%d" % (name, t.device.index, device))


def _device_of(t):
    return t.device.index if (t is not None and t.is_cuda) else None


def _remember(handle: int, **dims) -> int:
    with _dims_lock:
        _dims[handle] = dims
    return handle


def _recall(handle: int):
    return _dims.get(handle)


def _forget(handle: int) -> None:
    with _dims_lock:
        _dims.pop(handle, None)


def _check_io(handle: int, X, Y, M: int) -> None:
    d = _recall(handle)
    if d is not None:
        _same(X, "X", d["dt"], d.get("dev"))
        _same(Y, "Y", d["dt"], d.get("dev"))
    if d is not None and M > 0:
        _need(X, M * d["d_in"] * _esize(d["dt"]), "X")
        _need(Y, M * d["d_out"] * _esize(d["dt"]), "Y")


def _host_i32(a):
    if a is None:
        return None, None
    arr = np.ascontiguousarray(np.asarray(a), dtype=np.int32)
    return arr, arr.ctypes.data_as(_i32p)


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


def _check(fn: str, status: int):
    if status != PIFA_OK:
        raise PifaError(fn, status)


# ---------------------------------------------------------------- entry points
def pifa_status_string(status: int) -> str:
    return lib().pifa_status_string(int(status)).decode()


def pifa_gemm_plan(M: int, N: int, K: int, wide_epilogue: int = True):
    """(tile_m, tile_n, k_splits) of a prefill product of M x N outputs over K
    (host only).  Raises on an invalid size."""
    tm, tn, ks = _i64(), _i64(), _i64()
    _check("pifa_gemm_plan", lib().pifa_gemm_plan(int(M), int(N), int(K), int(wide_epilogue or 0), ctypes.byref(tm),
                                                  ctypes.byref(tn), ctypes.byref(ks)))
    return tm.value, tn.value, ks.value


def pifa_validate_partition(pivot_idx, nonpivot_idx, dims) -> int:
    """Returns the status code (no exception): PIFA_OK or the error."""
    piv, pp = _host_i32(pivot_idx)
    npv, npp = _host_i32(nonpivot_idx)
    return int(lib().pifa_validate_partition(pp, npp, pifa_dims(*dims)))


def pifa_layer_create(W_p, C, pivot_idx, nonpivot_idx, dims, dtype: int | None = None) -> int:
    """dims = (d_in, d_out, r); returns an opaque handle."""
    dt = _dtype_code(W_p) if dtype is None else int(dtype)
    piv, pp = _host_i32(pivot_idx)
    npv, npp = _host_i32(nonpivot_idx)
    d_in, d_out, r = (int(v) for v in dims)
    dev = _device_of(W_p)
    _same(W_p, "W_p", dt, dev)
    _same(C, "C", dt, dev)
    _need(W_p, r * d_in * _esize(dt), "W_p")
    _need(C, max(d_out - r, 0) * r * _esize(dt), "C")
    out = _vp()
    _check("pifa_layer_create", lib().pifa_layer_create(
        _dev_ptr(W_p, "W_p"), _dev_ptr(C, "C"), pp, npp, pifa_dims(*dims), dt, ctypes.byref(out)))
    return _remember(out.value, d_in=d_in, d_out=d_out, r=r, dt=dt, dev=dev)


def pifa_layer_destroy(handle: int) -> None:
    _forget(handle)
    _check("pifa_layer_destroy", lib().pifa_layer_destroy(handle))


def pifa_layer_reserve(handle: int, max_M: int) -> None:
    _check("pifa_layer_reserve", lib().pifa_layer_reserve(handle, int(max_M)))


def pifa_forward(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    _check_io(handle, X, Y, M)
    _check("pifa_forward", lib().pifa_forward(handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M,
                                              _stream(stream)))


def pifa_forward_noalloc(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    """pifa_forward with the library's fixed per-GPU scratch as workspace (no
    allocation; calls on one GPU must not overlap)."""
    M = X.shape[0] if M is None else int(M)
    _check_io(handle, X, Y, M)
    _check("pifa_forward_noalloc", lib().pifa_forward_noalloc(handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M,
                                                              _stream(stream)))


def pifa_layer_weight_bytes(handle: int) -> int:
    return int(lib().pifa_layer_weight_bytes(handle))


def pifa_layer_set_intermediate_scale(handle: int, log2_scale: int) -> None:
    _check("pifa_layer_set_intermediate_scale",
           lib().pifa_layer_set_intermediate_scale(handle, int(log2_scale)))


def pifa_layer_overflow_count(handle: int) -> int:
    out = _i64()
    _check("pifa_layer_overflow_count", lib().pifa_layer_overflow_count(handle, ctypes.byref(out)))
    return int(out.value)


def pifa_layer_backward(handle: int, X, Y, dY, dX=None, dW_p=None, dC=None, M: int | None = None,
                        stream=None) -> None:
    """Gradients of the layer: dX (bf16 M x d_in), dW_p (fp32 r x d_in), dC (fp32 (d_out-r) x r);
    each output may be None to skip it."""
    M = dY.shape[0] if M is None else int(M)
    d = _recall(handle)
    if d is not None:
        for t, name in ((X, "X"), (Y, "Y"), (dY, "dY"), (dX, "dX")):
            _same(t, name, PIFA_BF16, d.get("dev"))
        _same(dW_p, "dW_p", PIFA_F32, d.get("dev"))
        _same(dC, "dC", PIFA_F32, d.get("dev"))
    if d is not None and M > 0:  # bf16 activations and gradients, fp32 weight gradients
        for t, n, name in ((X, M * d["d_in"], "X"), (Y, M * d["d_out"], "Y"), (dY, M * d["d_out"], "dY"),
                           (dX, M * d["d_in"], "dX")):
            _need(t, 2 * n, name)
        _need(dW_p, 4 * d["r"] * d["d_in"], "dW_p")
        _need(dC, 4 * (d["d_out"] - d["r"]) * d["r"], "dC")
    _check("pifa_layer_backward", lib().pifa_layer_backward(
        handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), _dev_ptr(dY, "dY"), M, _dev_ptr(dX, "dX"),
        _dev_ptr(dW_p, "dW_p"), _dev_ptr(dC, "dC"), _stream(stream)))


def dense_forward(W, X, Y, M: int | None = None, d_in: int | None = None, d_out: int | None = None,
                  dtype: int | None = None, stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    d_in = W.shape[1] if d_in is None else int(d_in)
    d_out = W.shape[0] if d_out is None else int(d_out)
    dt = _dtype_code(W) if dtype is None else int(dtype)
    for t, name in ((W, "W"), (X, "X"), (Y, "Y")):
        _same(t, name, dt, _device_of(W))
    if M > 0:
        _need(W, d_out * d_in * _esize(dt), "W")
        _need(X, M * d_in * _esize(dt), "X")
        _need(Y, M * d_out * _esize(dt), "Y")
    _check("dense_forward", lib().dense_forward(_dev_ptr(W, "W"), _dev_ptr(X, "X"), _dev_ptr(Y, "Y"),
                                                M, d_in, d_out, dt, _stream(stream)))


def dense_layer_create(W, d_in: int | None = None, d_out: int | None = None,
                       dtype: int | None = None) -> int:
    d_in = W.shape[1] if d_in is None else int(d_in)
    d_out = W.shape[0] if d_out is None else int(d_out)
    dt = _dtype_code(W) if dtype is None else int(dtype)
    _same(W, "W", dt)
    _need(W, d_out * d_in * _esize(dt), "W")
    out = _vp()
    _check("dense_layer_create", lib().dense_layer_create(_dev_ptr(W, "W"), d_in, d_out, dt,
                                                          ctypes.byref(out)))
    return _remember(out.value, d_in=d_in, d_out=d_out, dt=dt, dev=_device_of(W))


def dense_layer_forward(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    _check_io(handle, X, Y, M)
    _check("dense_layer_forward", lib().dense_layer_forward(handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M,
                                                            _stream(stream)))


def dense_layer_reserve(handle: int, max_M: int) -> None:
    _check("dense_layer_reserve", lib().dense_layer_reserve(handle, int(max_M)))


def dense_layer_destroy(handle: int) -> None:
    _forget(handle)
    _check("dense_layer_destroy", lib().dense_layer_destroy(handle))


def lowrank_uv_forward(U, V, X, Y, M: int | None = None, dims=None, dtype: int | None = None,
                       stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    dims = (V.shape[1], U.shape[0], U.shape[1]) if dims is None else dims
    dt = _dtype_code(U) if dtype is None else int(dtype)
    d_in, d_out, r = (int(v) for v in dims)
    for t, name in ((U, "U"), (V, "V"), (X, "X"), (Y, "Y")):
        _same(t, name, dt, _device_of(U))
    if M > 0:
        _need(U, d_out * r * _esize(dt), "U")
        _need(V, r * d_in * _esize(dt), "V")
        _need(X, M * d_in * _esize(dt), "X")
        _need(Y, M * d_out * _esize(dt), "Y")
    _check("lowrank_uv_forward", lib().lowrank_uv_forward(
        _dev_ptr(U, "U"), _dev_ptr(V, "V"), _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M, pifa_dims(*dims),
        dt, _stream(stream)))


def lowrank_layer_create(U, V, dims=None, dtype: int | None = None) -> int:
    dims = (V.shape[1], U.shape[0], U.shape[1]) if dims is None else dims
    dt = _dtype_code(U) if dtype is None else int(dtype)
    d_in, d_out, r = (int(v) for v in dims)
    _same(U, "U", dt, _device_of(U))
    _same(V, "V", dt, _device_of(U))
    _need(U, d_out * r * _esize(dt), "U")
    _need(V, r * d_in * _esize(dt), "V")
    out = _vp()
    _check("lowrank_layer_create", lib().lowrank_layer_create(
        _dev_ptr(U, "U"), _dev_ptr(V, "V"), pifa_dims(*dims), dt, ctypes.byref(out)))
    return _remember(out.value, d_in=d_in, d_out=d_out, dt=dt, dev=_device_of(U))


def lowrank_layer_forward(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    _check_io(handle, X, Y, M)
    _check("lowrank_layer_forward", lib().lowrank_layer_forward(
        handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M, _stream(stream)))


def lowrank_layer_reserve(handle: int, max_M: int) -> None:
    _check("lowrank_layer_reserve", lib().lowrank_layer_reserve(handle, int(max_M)))


def lowrank_layer_destroy(handle: int) -> None:
    _forget(handle)
    _check("lowrank_layer_destroy", lib().lowrank_layer_destroy(handle))


def pifa_group_create(layers, dtype: int | None = None) -> int:
    """layers: sequence of (W_p, C, pivot_idx, nonpivot_idx, (d_in, d_out, r)) with one d_in;
    returns an opaque group handle."""
    n = len(layers)
    wp = (_vp * max(n, 1))()
    cc = (_vp * max(n, 1))()
    pp = (_i32p * max(n, 1))()
    npp = (_i32p * max(n, 1))()
    dims = (pifa_dims * max(n, 1))()
    keep = []
    dt = (_dtype_code(layers[0][0]) if n else PIFA_BF16) if dtype is None else int(dtype)
    dev = _device_of(layers[0][0]) if n else None
    for i, (W_p, C, piv, npiv, d) in enumerate(layers):
        if dt == PIFA_BF16:  # the only group dtype; the library rejects the others
            _same(W_p, "W_p", dt, dev)
            _same(C, "C", dt, dev)
            _need(W_p, int(d[2]) * int(d[0]) * 2, "W_p")
            _need(C, max(int(d[1]) - int(d[2]), 0) * int(d[2]) * 2, "C")
        wp[i] = _dev_ptr(W_p, "W_p")
        cc[i] = _dev_ptr(C, "C")
        a, ap = _host_i32(piv)
        b, bp = _host_i32(npiv)
        keep += [a, b]
        pp[i] = ap
        npp[i] = bp
        dims[i] = pifa_dims(*d)
    out = _vp()
    _check("pifa_group_create", lib().pifa_group_create(n, wp, cc, pp, npp, dims, dt, ctypes.byref(out)))
    return _remember(out.value, d_in=int(layers[0][4][0]), d_out=sum(int(l[4][1]) for l in layers), dt=dt,
                     dev=dev)


def pifa_group_destroy(handle: int) -> None:
    _forget(handle)
    _check("pifa_group_destroy", lib().pifa_group_destroy(handle))


def pifa_group_reserve(handle: int, max_M: int) -> None:
    _check("pifa_group_reserve", lib().pifa_group_reserve(handle, int(max_M)))


def pifa_group_forward(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    M = X.shape[0] if M is None else int(M)
    _check_io(handle, X, Y, M)
    _check("pifa_group_forward", lib().pifa_group_forward(handle, _dev_ptr(X, "X"), _dev_ptr(Y, "Y"), M,
                                                          _stream(stream)))


def pifa_group_weight_bytes(handle: int) -> int:
    return int(lib().pifa_group_weight_bytes(handle))


def pifa_group_set_intermediate_scale(handle: int, log2_scale: int) -> None:
    _check("pifa_group_set_intermediate_scale",
           lib().pifa_group_set_intermediate_scale(handle, int(log2_scale)))


def pifa_group_overflow_count(handle: int) -> int:
    out = _i64()
    _check("pifa_group_overflow_count", lib().pifa_group_overflow_count(handle, ctypes.byref(out)))
    return int(out.value)


def pifa_calib_create(d_in: int) -> int:
    out = _vp()
    _check("pifa_calib_create", lib().pifa_calib_create(int(d_in), ctypes.byref(out)))
    return _remember(out.value, n=int(d_in))


def pifa_calib_destroy(handle: int) -> None:
    _forget(handle)
    _check("pifa_calib_destroy", lib().pifa_calib_destroy(handle))


def pifa_calib_reset(handle: int, stream=None) -> None:
    _check("pifa_calib_reset", lib().pifa_calib_reset(handle, _stream(stream)))


def pifa_calib_accumulate(handle: int, X_o, X_u, B: int | None = None, stream=None) -> None:
    B = X_u.shape[0] if B is None else int(B)
    d = _recall(handle)
    if d is not None:
        _same(X_o, "X_o", PIFA_BF16)
        _same(X_u, "X_u", PIFA_BF16)
    if d is not None and B > 0:
        _need(X_o, 2 * B * d["n"], "X_o")
        _need(X_u, 2 * B * d["n"], "X_u")
    _check("pifa_calib_accumulate", lib().pifa_calib_accumulate(handle, _dev_ptr(X_o, "X_o"), _dev_ptr(X_u, "X_u"),
                                                                B, _stream(stream)))


def pifa_calib_read(handle: int, S=None, P=None, stream=None) -> None:
    d = _recall(handle)
    _same(S, "S", "f64")
    _same(P, "P", "f64")
    if d is not None:
        _need(S, 8 * d["n"] * d["n"], "S")
        _need(P, 8 * d["n"] * d["n"], "P")
    _check("pifa_calib_read", lib().pifa_calib_read(handle, _dev_ptr(S, "S"), _dev_ptr(P, "P"), _stream(stream)))


def pifa_calib_reconstruct(handle: int, W, Vt, lam: float, alpha: float, U_r=None, Vt_r=None, stream=None):
    """Returns (U_r, Vt_r) as device fp64 tensors (allocated when not given)."""
    import torch
    d_out, d_in = W.shape
    r = Vt.shape[0]
    if U_r is None:
        U_r = torch.empty((d_out, r), dtype=torch.float64, device=W.device)
    if Vt_r is None:
        Vt_r = torch.empty((r, d_in), dtype=torch.float64, device=W.device)
    for t, name in ((W, "W"), (Vt, "Vt"), (U_r, "U_r"), (Vt_r, "Vt_r")):
        _same(t, name, "f64", _device_of(W))
    d = _recall(handle)
    if d is not None:
        n = d["n"]
        for t, nb, name in ((W, d_out * n, "W"), (Vt, r * n, "Vt"), (U_r, d_out * r, "U_r"), (Vt_r, r * n, "Vt_r")):
            _need(t, 8 * nb, name)
    _check("pifa_calib_reconstruct", lib().pifa_calib_reconstruct(
        handle, _dev_ptr(W, "W"), int(d_out), _dev_ptr(Vt, "Vt"), int(r), float(lam), float(alpha),
        _dev_ptr(U_r, "U_r"), _dev_ptr(Vt_r, "Vt_r"), _stream(stream)))
    return U_r, Vt_r


def pifa_build_f64(W, r: int, stream=None):
    """Algorithm "Pivoting Factorization" on the GPU for a device fp64 W'
    (d_out x d_in).  Returns (pivot_idx, nonpivot_idx, W_p, C, report) with
    sorted numpy index arrays, device fp64 W_p / C, and the 4-entry report."""
    import torch
    if W.dtype != torch.float64:
        raise TypeError("W must be float64")
    d_out, d_in = W.shape
    r = int(r)
    Wp = torch.empty((r, d_in), dtype=torch.float64, device=W.device)
    C = torch.empty((d_out - r, r), dtype=torch.float64, device=W.device)
    piv = np.zeros(r, np.int32)
    npiv = np.zeros(max(d_out - r, 0), np.int32)
    report = (ctypes.c_double * 4)()
    npp = npiv.ctypes.data_as(_i32p) if npiv.size else None
    _check("pifa_build_f64", lib().pifa_build_f64(
        _dev_ptr(W, "W"), pifa_dims(d_in, d_out, r), _dev_ptr(Wp, "W_p"), C.data_ptr() if C.numel() else None,
        piv.ctypes.data_as(_i32p), npp, report, _stream(stream)))
    return piv, npiv, Wp, C, np.array(list(report))


# Buffers of the norms and 4-bit layers: every tensor given has the element
# type, lives on the device that is current (the kernels run there), is
# contiguous and holds what the call reads or writes; an input (`whole`) nothing
# besides, unless the caller gave the number of rows, and rows, where there is a
# dimension for them, are d values long.  `like`: a shape that is right as it is.
def _ptr_of(t, name: str, dtype, count: int, dev: int, whole: bool = False, d: int = 0, like=None) -> int | None:
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError("%s is %s, the call expects %s" % (name, t.dtype, dtype))
    if t.get_device() != dev:
        raise ValueError("%s is on %s, the call runs on cuda:%d" % (name, t.device, dev))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if like is None or t.shape != like:
        have = t.numel()
        if have != count and (whole or have < count):
            raise ValueError("%s holds %d values, the call needs %d" % (name, have, count))
        if d and t.dim() > 1 and t.shape[-1] != d:
            raise ValueError("%s is %s, its rows (last dimension) should hold %d values" % (name, tuple(t.shape), d))
    return t.data_ptr()


class _Torch:
    """What the calls below need of torch, looked up once: a decode step's calls
    are short, and torch.cuda.current_stream() alone takes longer than a launch."""

    def __init__(self):
        import torch
        self.empty, self.empty_like, self.zeros = torch.empty, torch.empty_like, torch.zeros
        self.bf16, self.f32, self.u8, self.e4m3 = torch.bfloat16, torch.float32, torch.uint8, torch.float8_e4m3fn
        self.i32 = torch.int32
        self.codes = {torch.bfloat16: PIFA_BF16, torch.float32: PIFA_F32}
        self.device = torch.cuda.current_device
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

    def stream(self, stream, dev: int) -> int:
        """The given stream, or the device's current one."""
        if stream is None and self.raw_stream is not None:
            return self.raw_stream(dev)
        if getattr(stream, "device_index", dev) != dev:
            raise ValueError("the stream is on cuda:%d, the call runs on cuda:%d" % (stream.device_index, dev))
        return _stream(stream)

    def under(self, stream):
        """Context in which a call's outputs and workspaces are allocated: the
        caching allocator hands a freed block out again on the stream it was
        allocated under at once, so that has to be the stream that uses it."""
        if stream is None:
            return contextlib.nullcontext()
        import torch
        raw = self.stream(stream, self.device())
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()
        return torch.cuda.stream(stream)

    def code(self, dtype) -> int:
        c = self.codes.get(dtype)
        if c is None:
            raise TypeError("unsupported dtype %s (bf16 or fp32)" % dtype)
        return c


_torch = None


def _rt() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _rows_of(t, name: str, M, d):
    """(M, d, whole, row, like) of a call on the rows of t: its own M and d, where
    not given, and what _ptr_of is to check of the others."""
    if M is None and d is None:
        like = t.shape
        if not like:
            raise ValueError("%s has no dimension" % name)
        d = like[-1]
        return t.numel() // max(d, 1), d, True, d, like
    d = t.shape[-1] if d is None else int(d)
    if M is not None:
        return int(M), d, False, 0, None
    n = t.numel()
    if d > 0 and n % d:
        raise ValueError("%s holds %d values, no whole rows of %d" % (name, n, d))
    return n // max(d, 1), d, True, 0, None


def rms_norm_forward(X, gain, eps: float, R=None, H=None, Y=None, M: int | None = None, d: int | None = None,
                     stream=None):
    """The norm of the rows of X + R (R may be None), times gain (may be None).
    Returns Y (allocated when not given); H, where given, takes X + R.  The
    rows are X's last dimension, or d values each where d is given; with M given,
    the first M rows of buffers that may hold more."""
    rt = _rt()
    M, d, whole, row, like = _rows_of(X, "X", M, d)
    if Y is None:
        with rt.under(stream):
            Y = rt.empty_like(X)
    dt, dev, n = X.dtype, rt.device(), M * d
    code = rt.code(dt)
    _check("rms_norm_forward", lib().rms_norm_forward(
        _ptr_of(X, "X", dt, n, dev, whole, 0, like), _ptr_of(R, "R", dt, n, dev, whole, row, like),
        _ptr_of(gain, "gain", dt, d, dev, True), eps, _ptr_of(H, "H", dt, n, dev, False, row, like),
        _ptr_of(Y, "Y", dt, n, dev, False, row, like), M, d, code, rt.stream(stream, dev)))
    return Y


def rms_norm_forward_e4m3(X, gain, eps: float, R=None, H=None, Q=None, scale=None, M: int | None = None,
                          d: int | None = None, stream=None):
    """The same norm in 8 bits.  Returns (Q, scale): float8_e4m3fn rows and one
    fp32 scale a row, which stand for Q * scale (allocated when not given)."""
    rt = _rt()
    M, d, whole, row, like = _rows_of(X, "X", M, d)
    if Q is None or scale is None:
        with rt.under(stream):
            Q = rt.empty(X.shape, dtype=rt.e4m3, device=X.device) if Q is None else Q
            scale = rt.empty(M, dtype=rt.f32, device=X.device) if scale is None else scale
    dt, dev, n = X.dtype, rt.device(), M * d
    code = rt.code(dt)
    _check("rms_norm_forward_e4m3", lib().rms_norm_forward_e4m3(
        _ptr_of(X, "X", dt, n, dev, whole, 0, like), _ptr_of(R, "R", dt, n, dev, whole, row, like),
        _ptr_of(gain, "gain", dt, d, dev, True), eps, _ptr_of(H, "H", dt, n, dev, False, row, like),
        _ptr_of(Q, "Q", rt.e4m3, n, dev, False, row, like),
        _ptr_of(scale, "scale", rt.f32, M, dev), M, d, code, rt.stream(stream, dev)))
    return Q, scale


def rms_norm_backward_bytes(M: int, d: int) -> int:
    return int(lib().rms_norm_backward_bytes(int(M), int(d)))


def rms_norm_backward(H, gain, dY, eps: float, dR=None, dX=None, dgain=None, work=None, M: int | None = None,
                      d: int | None = None, stream=None, need_dX: bool = True, need_dgain: bool = True):
    """Gradients of rms_norm_forward: (dX, dgain), dX plus dR where given.
    Outputs and workspace are allocated when not given, under the call's stream; need_dX / need_dgain
    False skip one (None in its place)."""
    rt = _rt()
    M, d, whole, row, like = _rows_of(H, "H", M, d)
    new_dX, new_dgain = dX is None and need_dX, dgain is None and need_dgain
    new_work = work is None and (new_dgain or dgain is not None)
    if new_dX or new_dgain or new_work:
        with rt.under(stream):
            dX = rt.empty_like(H) if new_dX else dX
            dgain = rt.empty(d, dtype=rt.f32, device=H.device) if new_dgain else dgain
            work = rt.empty(rms_norm_backward_bytes(M, d), dtype=rt.u8, device=H.device) if new_work else work
    dt, dev, n = H.dtype, rt.device(), M * d
    code = rt.code(dt)
    nwork = 0 if work is None else work.numel() * work.element_size()
    _check("rms_norm_backward", lib().rms_norm_backward(
        _ptr_of(H, "H", dt, n, dev, whole, 0, like), _ptr_of(gain, "gain", dt, d, dev, True),
        _ptr_of(dY, "dY", dt, n, dev, whole, row, like), _ptr_of(dR, "dR", dt, n, dev, whole, row, like), eps,
        _ptr_of(dX, "dX", dt, n, dev, False, row, like),
        _ptr_of(dgain, "dgain", rt.f32, d, dev), M, d, code,
        None if work is None else _ptr_of(work, "work", work.dtype, 0, dev), nwork, rt.stream(stream, dev)))
    return dX, dgain


def q4_layer_create(W, d_in: int | None = None, d_out: int | None = None, dtype: int | None = None) -> int:
    """Quantizes W (d_out x d_in) to 4 bits; returns an opaque handle."""
    rt = _rt()
    whole = d_in is None and d_out is None
    d_in = W.shape[1] if d_in is None else int(d_in)
    d_out = W.shape[0] if d_out is None else int(d_out)
    dt = _dtype_code(W) if dtype is None else int(dtype)
    dev = rt.device()
    out = _vp()
    _check("q4_layer_create", lib().q4_layer_create(_ptr_of(W, "W", _torch_dtype(dt), d_out * d_in, dev, whole), d_in,
                                                    d_out, dt, ctypes.byref(out)))
    return _remember(out.value, d_in=d_in, d_out=d_out, dt=PIFA_BF16, dev=dev)


def q4_layer_create_mx(codes, scales, d_in: int | None = None, d_out: int | None = None) -> int:
    """codes: uint8 d_out x d_in / 2 (the lower index in the lower half of a
    byte), scales: uint8 d_out x d_in / 32 (powers of two, biased by 127)."""
    rt = _rt()
    whole = d_in is None and d_out is None
    d_in = 2 * codes.shape[1] if d_in is None else int(d_in)
    d_out = codes.shape[0] if d_out is None else int(d_out)
    dev = rt.device()
    out = _vp()
    whole = whole and d_in % 32 == 0  # the library refuses others
    _check("q4_layer_create_mx", lib().q4_layer_create_mx(
        _ptr_of(codes, "codes", rt.u8, d_out * (d_in // 2), dev, whole),
        _ptr_of(scales, "scales", rt.u8, d_out * (d_in // 32), dev, whole, d_in // 32 if whole else 0), d_in, d_out,
        ctypes.byref(out)))
    return _remember(out.value, d_in=d_in, d_out=d_out, dt=PIFA_BF16, dev=dev)


def q4_layer_destroy(handle: int) -> None:
    _forget(handle)
    _check("q4_layer_destroy", lib().q4_layer_destroy(handle))


def q4_layer_read(handle: int, codes=None, scales=None, stream=None) -> None:
    """Copies the layer's codes and scales (either may be None)."""
    rt = _rt()
    d = _recall(handle) or {"d_in": 0, "d_out": 0}
    dev = rt.device()
    _check("q4_layer_read", lib().q4_layer_read(
        handle, _ptr_of(codes, "codes", rt.u8, d["d_out"] * d["d_in"] // 2, dev),
        _ptr_of(scales, "scales", rt.u8, d["d_out"] * d["d_in"] // 32, dev), rt.stream(stream, dev)))


def q4_layer_weight_bytes(handle: int) -> int:
    return int(lib().q4_layer_weight_bytes(handle))


def q4_layer_reserve(handle: int, max_M: int) -> None:
    _check("q4_layer_reserve", lib().q4_layer_reserve(handle, int(max_M)))


def _q4_rows(X, name: str, d_in: int, M):
    """Rows of a 4-bit layer's call: X's last dimension, where M is not given."""
    if M is not None:
        return int(M)
    if X.dim() == 0 or (d_in and X.shape[-1] != d_in):
        raise ValueError("%s is %s, its rows (last dimension) should hold %d values" % (name, tuple(X.shape), d_in))
    return X.numel() // d_in if d_in else X.shape[0]


def q4_layer_forward(handle: int, X, Y, M: int | None = None, stream=None) -> None:
    rt = _rt()
    d = _recall(handle) or {"d_in": 0, "d_out": 0}
    row = d["d_out"] if M is None else 0
    M = _q4_rows(X, "X", d["d_in"], M)
    dev = rt.device()
    _check("q4_layer_forward", lib().q4_layer_forward(
        handle, _ptr_of(X, "X", rt.bf16, M * d["d_in"], dev),
        _ptr_of(Y, "Y", rt.bf16, M * d["d_out"], dev, False, row), M, rt.stream(stream, dev)))


def q4_layer_forward_e4m3(handle: int, Q, scale, Y, M: int | None = None, stream=None) -> None:
    rt = _rt()
    d = _recall(handle) or {"d_in": 0, "d_out": 0}
    row = d["d_out"] if M is None else 0
    M = _q4_rows(Q, "Q", d["d_in"], M)
    dev = rt.device()
    _check("q4_layer_forward_e4m3", lib().q4_layer_forward_e4m3(
        handle, _ptr_of(Q, "Q", rt.e4m3, M * d["d_in"], dev), _ptr_of(scale, "scale", rt.f32, M, dev),
        _ptr_of(Y, "Y", rt.bf16, M * d["d_out"], dev, False, row), M, rt.stream(stream, dev)))


def q4_layer_norm_forward(handle: int, X, gain, eps: float, R=None, H=None, Y=None, M: int | None = None,
                          stream=None) -> None:
    rt = _rt()
    d = _recall(handle) or {"d_in": 0, "d_out": 0}
    row_in, row_out, whole, like = (d["d_in"], d["d_out"], d["d_in"] > 0, X.shape) if M is None else (0, 0, False, None)
    M = _q4_rows(X, "X", d["d_in"], M)
    dev, bf, n = rt.device(), rt.bf16, M * d["d_in"]
    _check("q4_layer_norm_forward", lib().q4_layer_norm_forward(
        handle, _ptr_of(X, "X", bf, n, dev), _ptr_of(R, "R", bf, n, dev, whole, row_in, like),
        _ptr_of(gain, "gain", bf, d["d_in"], dev, d["d_in"] > 0), eps, _ptr_of(H, "H", bf, n, dev, False, row_in, like),
        _ptr_of(Y, "Y", bf, M * d["d_out"], dev, False, row_out), M, rt.stream(stream, dev)))


def layer_norm_forward(X, gain, bias, eps: float, R=None, H=None, Y=None, M: int | None = None, d: int | None = None,
                       stream=None):
    """The layer norm of the rows of X + R (R may be None), times gain plus bias
    (either may be None).  Returns Y (allocated when not given); H, where given,
    takes X + R.  Rows, M and d as for rms_norm_forward."""
    rt = _rt()
    M, d, whole, row, like = _rows_of(X, "X", M, d)
    if Y is None:
        with rt.under(stream):
            Y = rt.empty_like(X)
    dt, dev, n = X.dtype, rt.device(), M * d
    code = rt.code(dt)
    _check("layer_norm_forward", lib().layer_norm_forward(
        _ptr_of(X, "X", dt, n, dev, whole, 0, like), _ptr_of(R, "R", dt, n, dev, whole, row, like),
        _ptr_of(gain, "gain", dt, d, dev, True), _ptr_of(bias, "bias", dt, d, dev, True), eps,
        _ptr_of(H, "H", dt, n, dev, False, row, like), _ptr_of(Y, "Y", dt, n, dev, False, row, like), M, d, code,
        rt.stream(stream, dev)))
    return Y


def layer_norm_backward_bytes(M: int, d: int) -> int:
    return int(lib().layer_norm_backward_bytes(int(M), int(d)))


def layer_norm_backward(H, gain, dY, eps: float, dR=None, dX=None, dgain=None, dbias=None, work=None,
                        M: int | None = None, d: int | None = None, stream=None, need_dX: bool = True,
                        need_dgain: bool = True, need_dbias: bool = True):
    """Gradients of layer_norm_forward: (dX, dgain, dbias), dX plus dR where given.
    Outputs and workspace are allocated when not given, under the call's stream;
    need_dX / need_dgain / need_dbias False skip one (None in its place)."""
    rt = _rt()
    M, d, whole, row, like = _rows_of(H, "H", M, d)
    new_dX, new_dgain, new_dbias = dX is None and need_dX, dgain is None and need_dgain, dbias is None and need_dbias
    new_work = work is None and (new_dgain or new_dbias or dgain is not None or dbias is not None)
    if new_dX or new_dgain or new_dbias or new_work:
        with rt.under(stream):
            dX = rt.empty_like(H) if new_dX else dX
            dgain = rt.empty(d, dtype=rt.f32, device=H.device) if new_dgain else dgain
            dbias = rt.empty(d, dtype=rt.f32, device=H.device) if new_dbias else dbias
            work = rt.empty(layer_norm_backward_bytes(M, d), dtype=rt.u8, device=H.device) if new_work else work
    dt, dev, n = H.dtype, rt.device(), M * d
    code = rt.code(dt)
    nwork = 0 if work is None else work.numel() * work.element_size()
    _check("layer_norm_backward", lib().layer_norm_backward(
        _ptr_of(H, "H", dt, n, dev, whole, 0, like), _ptr_of(gain, "gain", dt, d, dev, True),
        _ptr_of(dY, "dY", dt, n, dev, whole, row, like), _ptr_of(dR, "dR", dt, n, dev, whole, row, like), eps,
        _ptr_of(dX, "dX", dt, n, dev, False, row, like), _ptr_of(dgain, "dgain", rt.f32, d, dev),
        _ptr_of(dbias, "dbias", rt.f32, d, dev), M, d, code,
        None if work is None else _ptr_of(work, "work", work.dtype, 0, dev), nwork, rt.stream(stream, dev)))
    return dX, dgain, dbias


def adapter_plan_bytes(M: int, n: int) -> int:
    return int(lib().adapter_plan_bytes(int(M), int(n)))


def adapter_plan(ids, n: int, plan, stream=None) -> None:
    """Sorts the rows of a batch by their adapters, ids (int32, one a row; outside
    [0, n): none), into plan (uint8, adapter_plan_bytes(M, n)).  See AdapterPlan."""
    rt = _rt()
    dev, M, n = rt.device(), ids.numel(), int(n)
    _check("adapter_plan", lib().adapter_plan(_ptr_of(ids, "ids", rt.i32, M, dev, True), M, n,
                                              _ptr_of(plan, "plan", rt.u8, 0, dev), plan.numel(),
                                              rt.stream(stream, dev)))


def adapter_forward_bytes(M: int, d_in: int, d_out: int, r: int, n: int) -> int:
    return int(lib().adapter_forward_bytes(int(M), int(d_in), int(d_out), int(r), int(n)))


def adapter_backward_bytes(M: int, d_in: int, d_out: int, r: int, n: int) -> int:
    return int(lib().adapter_backward_bytes(int(M), int(d_in), int(d_out), int(r), int(n)))


def _adapter_dims(A, B, plan):
    """(M, d_in, d_out, r, n) of a call with these weights and this plan."""
    if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
        raise ValueError("A is %s, B %s: n x r x d_in and n x d_out x r are expected" % (tuple(A.shape), tuple(B.shape)))
    if plan.n != A.shape[0]:
        raise ValueError("the plan is for %d adapters, A holds %d" % (plan.n, A.shape[0]))
    return plan.M, A.shape[2], B.shape[1], A.shape[1], plan.n


def adapter_forward(X, A, B, plan, scale=None, Y0=None, Y=None, work=None, stream=None):
    """Y0 (may be None: zeros) plus each row's adapter: scale (X A^T) B^T.  A is n x r
    x d_in, B n x d_out x r, plan an AdapterPlan of the rows' ids.  Returns Y
    (allocated when not given; may be Y0).  Rows are the last dimension."""
    rt = _rt()
    M, d_in, d_out, r, n = _adapter_dims(A, B, plan)
    dev, bf = rt.device(), rt.bf16
    if Y is None or work is None:
        with rt.under(stream):
            Y = rt.empty((*X.shape[:-1], d_out), dtype=bf, device=X.device) if Y is None else Y
            work = rt.empty(adapter_forward_bytes(M, d_in, d_out, r, n), dtype=rt.u8, device=X.device) if work is None else work
    _check("adapter_forward", lib().adapter_forward(
        _ptr_of(X, "X", bf, M * d_in, dev, True, d_in), _ptr_of(A, "A", bf, n * r * d_in, dev, True),
        _ptr_of(B, "B", bf, n * r * d_out, dev, True), _ptr_of(scale, "scale", rt.f32, n, dev, True), plan.pointer(dev),
        _ptr_of(Y0, "Y0", bf, M * d_out, dev, True, d_out), _ptr_of(Y, "Y", bf, M * d_out, dev, False, d_out), M, d_in,
        d_out, r, n, _ptr_of(work, "work", rt.u8, 0, dev), work.numel(), rt.stream(stream, dev)))
    return Y


def adapter_backward(X, A, B, plan, dY, scale=None, dX0=None, dX=None, dA=None, dB=None, work=None, stream=None,
                     need_dX: bool = True, need_dA: bool = True, need_dB: bool = True):
    """Gradients of adapter_forward: (dX, dA, dB), dX plus dX0 where given (dX may be
    dX0), dA and dB in fp32.  Outputs and workspace are allocated when not given,
    under the call's stream; need_dX / need_dA / need_dB False skip one (None in
    its place)."""
    rt = _rt()
    M, d_in, d_out, r, n = _adapter_dims(A, B, plan)
    dev, bf, f32 = rt.device(), rt.bf16, rt.f32
    new_dX, new_dA, new_dB = dX is None and need_dX, dA is None and need_dA, dB is None and need_dB
    if new_dX or new_dA or new_dB or work is None:
        with rt.under(stream):
            dX = rt.empty_like(X) if new_dX else dX
            dA = rt.empty(A.shape, dtype=f32, device=A.device) if new_dA else dA
            dB = rt.empty(B.shape, dtype=f32, device=B.device) if new_dB else dB
            work = rt.empty(adapter_backward_bytes(M, d_in, d_out, r, n), dtype=rt.u8, device=X.device) if work is None else work
    _check("adapter_backward", lib().adapter_backward(
        _ptr_of(X, "X", bf, M * d_in, dev, True, d_in), _ptr_of(A, "A", bf, n * r * d_in, dev, True),
        _ptr_of(B, "B", bf, n * r * d_out, dev, True), _ptr_of(scale, "scale", f32, n, dev, True), plan.pointer(dev),
        _ptr_of(dY, "dY", bf, M * d_out, dev, True, d_out), _ptr_of(dX0, "dX0", bf, M * d_in, dev, True, d_in),
        _ptr_of(dX, "dX", bf, M * d_in, dev, False, d_in), _ptr_of(dA, "dA", f32, n * r * d_in, dev, True),
        _ptr_of(dB, "dB", f32, n * r * d_out, dev, True), M, d_in, d_out, r, n, _ptr_of(work, "work", rt.u8, 0, dev),
        work.numel(), rt.stream(stream, dev)))
    return dX, dA, dB


def adamw_create(params, grads, states, weight_decay=0.0, copies=None, seed: int = 0) -> int:
    """A handle for one step of many tensors: params (fp32), grads (all fp32 or all
    bf16), states (m, v) in fp32 or (m, v, m_scale, v_scale) in 8 bits
    (float8_e4m3fn codes, uint8 scales, one for each 32 values), copies: bf16
    tensors (or None each) that take the parameters.  weight_decay: one for all
    or one each.  The tensors have to live as long as the handle (see AdamW)."""
    rt = _rt()
    params, grads, states = list(params), list(grads), [tuple(s) for s in states]
    count = len(params)
    copies = [None] * count if copies is None else list(copies)
    decay = [float(w) for w in weight_decay] if hasattr(weight_decay, "__len__") else [float(weight_decay)] * count
    if not count == len(grads) == len(states) == len(copies) == len(decay):
        raise ValueError("%d params, %d grads, %d states, %d copies, %d decays" % (count, len(grads), len(states),
                                                                                   len(copies), len(decay)))
    bits = 8 if states and len(states[0]) == 4 else 32
    g_type = grads[0].dtype if grads else rt.f32
    code, dev = rt.code(g_type), rt.device()
    table = (adamw_tensor * max(count, 1))()
    for t, p, g, s, c, w in zip(table, params, grads, states, copies, decay):
        if len(s) != (4 if bits == 8 else 2):
            raise ValueError("states are (m, v) of every tensor, or (m, v, m_scale, v_scale)")
        n, groups = p.numel(), -(-p.numel() // 32)
        kind = rt.e4m3 if bits == 8 else rt.f32
        t.p, t.g = _ptr_of(p, "params", rt.f32, n, dev, True), _ptr_of(g, "grads", g_type, n, dev, True)
        t.m, t.v = _ptr_of(s[0], "m", kind, n, dev, True), _ptr_of(s[1], "v", kind, n, dev, True)
        if bits == 8:
            t.m_scale = _ptr_of(s[2], "m_scale", rt.u8, groups, dev, True)
            t.v_scale = _ptr_of(s[3], "v_scale", rt.u8, groups, dev, True)
        t.p_bf16, t.n, t.weight_decay = _ptr_of(c, "copies", rt.bf16, n, dev, True), n, w
    out = _vp()
    _check("adamw_create", lib().adamw_create(table, count, bits, code, int(seed) & 0xFFFFFFFF, ctypes.byref(out)))
    return out.value


def adamw_destroy(handle: int) -> None:
    _check("adamw_destroy", lib().adamw_destroy(handle))


def adamw_step(handle: int, lr: float, beta1: float, beta2: float, eps: float, step: int = 0, grad_scale=None,
               stream=None) -> None:
    """One step.  step: its number, from 1 on; 0: the handle counts on the device.
    grad_scale: a device fp32 value that multiplies the gradients."""
    rt = _rt()
    dev = rt.device()
    _check("adamw_step", lib().adamw_step(handle, lr, beta1, beta2, eps, int(step),
                                          _ptr_of(grad_scale, "grad_scale", rt.f32, 1, dev, True),
                                          rt.stream(stream, dev)))


def adamw_count(handle: int) -> int:
    """Number of the handle's last step."""
    out = _i64()
    _check("adamw_count", lib().adamw_count(handle, ctypes.byref(out)))
    return int(out.value)


def pifa_probe_mfma(iters: int = 20000, stream=None):
    """(dense bf16 MFMA TFLOP/s, shader clock in MHz) of an MFMA-only kernel."""
    tf, mhz = ctypes.c_double(), ctypes.c_double()
    _check("pifa_probe_mfma", lib().pifa_probe_mfma(int(iters), ctypes.byref(tf), ctypes.byref(mhz),
                                                    _stream(stream)))
    return tf.value, mhz.value


def pifa_probe_mfma_random(iters: int = 20000, stream=None):
    """(dense bf16 MFMA TFLOP/s, shader clock in MHz) of an MFMA-only kernel
    whose operands change with every MFMA (random bf16 values)."""
    tf, mhz = ctypes.c_double(), ctypes.c_double()
    _check("pifa_probe_mfma_random", lib().pifa_probe_mfma_random(int(iters), ctypes.byref(tf), ctypes.byref(mhz),
                                                                  _stream(stream)))
    return tf.value, mhz.value


def pifa_probe_hbm_read(buf, reps: int = 5, stream=None) -> float:
    """GB/s of `reps` streaming reads of the device tensor `buf`."""
    nbytes = (buf.numel() * buf.element_size()) // 16 * 16
    out = ctypes.c_double()
    _check("pifa_probe_hbm_read", lib().pifa_probe_hbm_read(_dev_ptr(buf, "buf"), nbytes, int(reps),
                                                            ctypes.byref(out), _stream(stream)))
    return out.value


def pifa_profile_enable(on: bool) -> None:
    _check("pifa_profile_enable", lib().pifa_profile_enable(1 if on else 0))


def pifa_profile_reset() -> None:
    _check("pifa_profile_reset", lib().pifa_profile_reset())


def pifa_profile_read(max_sites: int = 64) -> dict:
    """{site name: (launches, total milliseconds)} since the last reset."""
    names = (ctypes.c_char_p * max_sites)()
    launches = (_i64 * max_sites)()
    ms = (ctypes.c_double * max_sites)()
    n = ctypes.c_int()
    _check("pifa_profile_read", lib().pifa_profile_read(names, launches, ms, max_sites, ctypes.byref(n)))
    return {names[i].decode(): (int(launches[i]), float(ms[i])) for i in range(n.value)}


# ---------------------------------------------------------------- convenience
class PifaLayer:
    """Owns a pifa_handle; ``layer(X)`` allocates Y and runs pifa_forward."""

    def __init__(self, W_p, C, pivot_idx, nonpivot_idx, d_out: int):
        self.d_in = int(W_p.shape[1])
        self.r = int(W_p.shape[0])
        self.d_out = int(d_out)
        self.dtype = W_p.dtype
        self.handle = pifa_layer_create(W_p, C, pivot_idx, nonpivot_idx, (self.d_in, self.d_out, self.r))

    def __call__(self, X, Y=None, stream=None):
        import torch
        if Y is None:
            Y = torch.empty((X.shape[0], self.d_out), dtype=X.dtype, device=X.device)
        pifa_forward(self.handle, X, Y, X.shape[0], stream)
        return Y

    def close(self):
        if self.handle:
            pifa_layer_destroy(self.handle)
            self.handle = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Q4Layer:
    """Owns a 4-bit layer: ``layer(X)`` allocates Y and runs q4_layer_forward.
    Rows are the last dimension of X (d_in values each) and of Y (d_out)."""

    def __init__(self, W=None, handle: int = 0, d_in: int = 0, d_out: int = 0):
        self.handle = q4_layer_create(W) if W is not None else handle
        self.d_in = int(W.shape[1]) if W is not None else int(d_in)
        self.d_out = int(W.shape[0]) if W is not None else int(d_out)

    @classmethod
    def from_mx(cls, codes, scales):
        """A layer of weights already in the format (see q4_layer_create_mx)."""
        return cls(None, q4_layer_create_mx(codes, scales), 2 * codes.shape[1], codes.shape[0])

    def _out(self, Y, X, stream):
        if Y is not None:
            return Y
        rt = _rt()
        with rt.under(stream):
            return rt.empty((*X.shape[:-1], self.d_out), dtype=rt.bf16, device=X.device)

    def __call__(self, X, Y=None, stream=None):
        Y = self._out(Y, X, stream)
        q4_layer_forward(self.handle, X, Y, None, stream)
        return Y

    def forward_e4m3(self, Q, scale, Y=None, stream=None):
        """Rows in 8 bits with a scale each, as rms_norm_forward_e4m3 returns them."""
        Y = self._out(Y, Q, stream)
        q4_layer_forward_e4m3(self.handle, Q, scale, Y, None, stream)
        return Y

    def norm_forward(self, X, gain, eps: float, R=None, H=None, Y=None, stream=None):
        """The product of the norm of X + R; H, where given, takes X + R.  Normed
        rows are rounded to bf16 from 9 of them on.  Calls that use the layer's
        workspace (see q4_layer_norm_forward in include/pifa.h) must not overlap."""
        Y = self._out(Y, X, stream)
        q4_layer_norm_forward(self.handle, X, gain, eps, R, H, Y, None, stream)
        return Y

    def reserve(self, max_M: int):
        q4_layer_reserve(self.handle, max_M)

    def read(self):
        """(codes, scales) as from_mx takes them."""
        import torch
        dev = "cuda:%d" % _rt().device()
        codes = torch.empty((self.d_out, self.d_in // 2), dtype=torch.uint8, device=dev)
        scales = torch.empty((self.d_out, self.d_in // 32), dtype=torch.uint8, device=dev)
        q4_layer_read(self.handle, codes, scales)
        return codes, scales

    def close(self):
        if self.handle:
            q4_layer_destroy(self.handle)
            self.handle = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdapterPlan:
    """The rows of a batch, sorted by adapter: ``AdapterPlan(ids, n)`` for the layers of
    one batch, ``update(ids)`` for the next one of as many rows (in the same
    memory, so that a captured graph may hold it)."""

    def __init__(self, ids, n: int, stream=None):
        rt = _rt()
        self.M, self.n = ids.numel(), int(n)
        with rt.under(stream):
            self.buffer = rt.empty(adapter_plan_bytes(self.M, self.n), dtype=rt.u8, device=ids.device)
        self.update(ids, stream)

    def update(self, ids, stream=None):
        if ids.numel() != self.M:
            raise ValueError("the plan is for %d rows, ids holds %d" % (self.M, ids.numel()))
        adapter_plan(ids, self.n, self.buffer, stream)

    def pointer(self, dev: int) -> int:
        return _ptr_of(self.buffer, "plan", self.buffer.dtype, 0, dev)


class AdamW:
    """Owns an AdamW handle and the tensors it points to.  Without states they are
    zeros, in 8 bits with bits=8; ``states`` holds them, (m, v) or (m, v, m_scale,
    v_scale) a tensor, and has to be of the ``bits`` that are asked for, if any are."""

    def __init__(self, params, grads, weight_decay=0.0, bits: int | None = None, copies=None, states=None, seed: int = 0):
        rt = _rt()
        self.handle = 0
        if bits not in (None, 8, 32):
            raise ValueError("bits is %r: 8 or 32" % (bits,))
        self.params, self.grads = list(params), list(grads)
        self.copies = None if copies is None else list(copies)
        if states is None:
            zeros = lambda p, dtype, n: rt.zeros(n, dtype=dtype, device=p.device)
            if bits != 8:
                states = [(rt.zeros(p.shape, dtype=rt.f32, device=p.device), rt.zeros(p.shape, dtype=rt.f32, device=p.device))
                          for p in self.params]
            else:
                states = [tuple(rt.zeros(p.shape, dtype=rt.u8, device=p.device).view(rt.e4m3) for _ in range(2)) +
                          tuple(zeros(p, rt.u8, -(-p.numel() // 32)) for _ in range(2)) for p in self.params]
        self.states = [tuple(s) for s in states]
        if bits and any(len(s) != (4 if bits == 8 else 2) for s in self.states):
            raise ValueError("states are not those of %d bits" % bits)
        self.handle = adamw_create(self.params, self.grads, self.states, weight_decay, self.copies, seed)

    def step(self, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, step: int = 0,
             grad_scale=None, stream=None):
        adamw_step(self.handle, lr, beta1, beta2, eps, step, grad_scale, stream)

    def count(self) -> int:
        return adamw_count(self.handle)

    def close(self):
        if self.handle:
            adamw_destroy(self.handle)
            self.handle = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
