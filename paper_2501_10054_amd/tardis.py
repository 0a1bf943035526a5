"""Thin ctypes binding of libtardis (include/tardis.h).

Argument marshalling only: every step of the method runs in the library's HIP
kernels.  Tensors are torch CUDA tensors used as plain device buffers; the
current torch stream is passed unless one is given.  Inference only: results carry no
gradient, also where operands ask for one.  The library must have been
built (``python -m paper_2501_10054_amd.build``); there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("TARDIS_LIB") or os.path.join(_HERE, "libtardis.so")

OK, ERR_INVALID_ARG, ERR_SHAPE, ERR_DTYPE, ERR_STATE, ERR_OOM, ERR_HIP = range(7)
ACT = {"gelu_erf": 0, "gelu_tanh": 1, "relu": 2, "identity": 3}
F32, BF16, FP8_E4M3 = 0, 1, 2
_TORCH_DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
_DTYPE_CODE = {torch.float32: F32, torch.bfloat16: BF16}

EXPORTS = (
    "tardis_calibrate", "tardis_calibrate_search", "tardis_estimate_errors", "tardis_assign_thresholds", "tardis_fold", "tardis_ffn_forward", "tardis_ffn_forward_batched",
    "tardis_ffn_forward_static", "tardis_stack_forward", "tardis_dense_forward", "tardis_get_folded", "tardis_get_predictor_state",
    "tardis_get_sketch_groups", "tardis_get_last_outliers", "tardis_get_last_union", "tardis_get_handover", "tardis_set_next_layer",
    "tardis_linear", "tardis_linear_workspace", "tardis_grouped_linear", "tardis_grouped_linear_workspace", "tardis_moe_route", "tardis_moe_route_workspace", "tardis_moe_combine",
    "tardis_rms_norm", "tardis_fp8_rows", "tardis_linear_fp8", "tardis_linear_fp8_workspace", "tardis_linear_4bit", "tardis_linear_4bit_workspace",
    "tardis_destroy", "tardis_release_memory", "tardis_status_string", "tardis_version",
)


class TardisError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class tardis_ffn_desc(C.Structure):
    _fields_ = [("d", C.c_int64), ("h", C.c_int64), ("dtype", C.c_int32), ("act", C.c_int32),
                ("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p)]


class tardis_fold_opts(C.Structure):
    _fields_ = [("sketch_bits", C.c_int32), ("folded_dtype", C.c_int32), ("max_batch", C.c_int64),
                ("deterministic", C.c_int32), ("margin", C.c_float)]


class tardis_linear_desc(C.Structure):
    _fields_ = [("n_in", C.c_int64), ("n_out", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("act", C.c_int32),
                ("reserved", C.c_int32), ("W", C.c_void_p), ("b", C.c_void_p)]


class tardis_norm_desc(C.Structure):
    _fields_ = [("d", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32), ("weight", C.c_void_p)]


class tardis_linear_fp8_desc(C.Structure):
    _fields_ = [("n_in", C.c_int64), ("n_out", C.c_int64), ("out_dtype", C.c_int32), ("act", C.c_int32), ("W", C.c_void_p), ("W_scales", C.c_void_p),
                ("b", C.c_void_p)]


class tardis_linear_4bit_desc(C.Structure):
    _fields_ = [("n_in", C.c_int64), ("n_out", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("act", C.c_int32), ("group", C.c_int32),
                ("W", C.c_void_p), ("scales", C.c_void_p), ("zeros", C.c_void_p), ("b", C.c_void_p)]


_lib_handle = None


def lib() -> C.CDLL:
    """The loaded shared library (loaded on first use)."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2501_10054_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i64, f32 = C.c_void_p, C.c_int64, C.c_float
        L.tardis_calibrate.argtypes = [C.POINTER(tardis_ffn_desc), vp, i64, f32, vp, vp, vp, vp, vp, vp]
        L.tardis_calibrate_search.argtypes = [C.POINTER(tardis_ffn_desc), vp, i64, f32, vp, f32, vp, vp, vp, vp, vp]
        L.tardis_estimate_errors.argtypes = [C.POINTER(tardis_ffn_desc), vp, i64, vp, vp, vp, vp, vp, vp, vp]
        L.tardis_assign_thresholds.argtypes = [vp, i64, f32, f32, f32, vp, vp]
        L.tardis_fold.argtypes = [C.POINTER(tardis_ffn_desc), vp, vp, vp, vp, C.POINTER(tardis_fold_opts), vp,
                                  C.POINTER(vp)]
        L.tardis_ffn_forward.argtypes = [vp, vp, vp, vp]
        L.tardis_ffn_forward_batched.argtypes = [vp, vp, i64, vp, vp]
        L.tardis_ffn_forward_static.argtypes = [vp, vp, i64, vp, vp, vp]
        L.tardis_dense_forward.argtypes = [vp, vp, i64, vp, vp]
        L.tardis_stack_forward.argtypes = [C.POINTER(vp), C.c_int32, vp, i64, vp, vp]
        L.tardis_set_next_layer.argtypes = [vp, vp]
        L.tardis_get_folded.argtypes = [vp, vp, vp, vp]
        L.tardis_get_predictor_state.argtypes = [vp, vp, vp, vp, vp]
        L.tardis_get_sketch_groups.argtypes = [vp, vp, vp]
        L.tardis_get_last_outliers.argtypes = [vp, i64, vp, vp, vp, vp]
        L.tardis_get_last_union.argtypes = [vp, i64, vp, vp, vp]
        L.tardis_get_handover.argtypes = [vp, i64, vp, vp]
        L.tardis_linear.argtypes = [C.POINTER(tardis_linear_desc), vp, i64, i64, vp, vp, vp, i64, vp]
        L.tardis_linear_workspace.argtypes = [C.POINTER(tardis_linear_desc), vp, i64, i64, C.POINTER(i64)]
        L.tardis_grouped_linear.argtypes = [C.POINTER(tardis_linear_desc), i64, vp, i64, i64, vp, vp, i64, i64, vp, vp, i64, vp]
        L.tardis_grouped_linear_workspace.argtypes = [C.POINTER(tardis_linear_desc), i64, vp, i64, i64, C.c_int32, i64, C.POINTER(i64)]
        L.tardis_moe_route.argtypes = [vp, i64, i64, i64, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, i64, vp]
        L.tardis_moe_route_workspace.argtypes = [i64, i64, i64, C.POINTER(i64)]
        L.tardis_moe_combine.argtypes = [vp, i64, vp, vp, i64, i64, i64, C.c_int32, vp, vp, C.c_int32, vp]
        norm, fp8, four = C.POINTER(tardis_norm_desc), C.POINTER(tardis_linear_fp8_desc), C.POINTER(tardis_linear_4bit_desc)
        L.tardis_rms_norm.argtypes = [norm, vp, i64, i64, vp, vp, vp, vp, vp]
        L.tardis_fp8_rows.argtypes = [vp, i64, i64, i64, C.c_int32, vp, vp, vp]
        L.tardis_linear_fp8.argtypes = [fp8, vp, vp, i64, i64, vp, vp, vp, i64, vp]
        L.tardis_linear_fp8_workspace.argtypes = [fp8, vp, i64, i64, C.POINTER(i64)]
        L.tardis_linear_4bit.argtypes = [four, vp, i64, i64, vp, vp, vp, i64, vp]
        L.tardis_linear_4bit_workspace.argtypes = [four, i64, i64, C.POINTER(i64)]
        L.tardis_destroy.argtypes = [vp]
        L.tardis_release_memory.argtypes = []
        L.tardis_status_string.argtypes = [C.c_int]
        L.tardis_status_string.restype = C.c_char_p
        L.tardis_version.argtypes = []
        L.tardis_version.restype = C.c_int32
        for name in EXPORTS:
            if name not in ("tardis_status_string", "tardis_version"):
                getattr(L, name).restype = C.c_int
        _lib_handle = L
    return _lib_handle


def status_string(status: int) -> str:
    return lib().tardis_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise TardisError(status, where)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# The handle of a device's current stream without the object that torch.cuda.current_stream() makes of it, which takes 3 of the 8 us of a
# small call.  Not torch's public interface, so the public call where it is missing
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return C.c_void_p(_raw_stream(_device()))
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


class FFN:
    """Device tensors of one FFN layer plus the matching C descriptor."""

    def __init__(self, W1, W2, b1=None, b2=None, act: str = "gelu_erf"):
        h, d = W1.shape
        assert W2.shape == (d, h)
        for t in (W1, W2, b1, b2):
            assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == W1.dtype)
        self.W1, self.W2, self.b1, self.b2 = W1, W2, b1, b2
        self.d, self.h, self.act = d, h, act
        self.dtype = _DTYPE_CODE[W1.dtype]
        self.desc = tardis_ffn_desc(d, h, self.dtype, ACT[act], W1.data_ptr(),
                                    b1.data_ptr() if b1 is not None else None, W2.data_ptr(),
                                    b2.data_ptr() if b2 is not None else None)


def tardis_calibrate(ffn: FFN, X_cal, coverage: float = 0.95, coverage_per_neuron=None, stream=None):
    """-> (lo, hi, a, c), four float32 device tensors of length h."""
    assert X_cal.is_cuda and X_cal.is_contiguous() and X_cal.dtype == ffn.W1.dtype and X_cal.shape[1] == ffn.d
    out = [torch.empty(ffn.h, dtype=torch.float32, device=X_cal.device) for _ in range(4)]
    st = lib().tardis_calibrate(C.byref(ffn.desc), _ptr(X_cal), X_cal.shape[0], float(coverage),
                                _ptr(coverage_per_neuron), *[_ptr(t) for t in out], _stream(stream))
    _check(st, "tardis_calibrate")
    return tuple(out)


def tardis_calibrate_search(ffn: FFN, X_cal, coverage: float = 0.95, step: float = 0.05, coverage_per_neuron=None,
                            stream=None):
    """-> (lo, hi, a, c) with greedily searched ranges."""
    assert X_cal.is_cuda and X_cal.is_contiguous() and X_cal.dtype == ffn.W1.dtype and X_cal.shape[1] == ffn.d
    out = [torch.empty(ffn.h, dtype=torch.float32, device=X_cal.device) for _ in range(4)]
    st = lib().tardis_calibrate_search(C.byref(ffn.desc), _ptr(X_cal), X_cal.shape[0], float(coverage),
                                       _ptr(coverage_per_neuron), float(step), *[_ptr(t) for t in out],
                                       _stream(stream))
    _check(st, "tardis_calibrate_search")
    return tuple(out)


def tardis_estimate_errors(ffn: FFN, X_cal, lo, hi, a, c, stream=None):
    """-> (err_neurons float32[h], err_layer float32[1]): empirical approximation error over X_cal."""
    err = torch.empty(ffn.h, dtype=torch.float32, device=X_cal.device)
    tot = torch.empty(1, dtype=torch.float32, device=X_cal.device)
    st = lib().tardis_estimate_errors(C.byref(ffn.desc), _ptr(X_cal), X_cal.shape[0], _ptr(lo), _ptr(hi), _ptr(a), _ptr(c),
                                      _ptr(err), _ptr(tot), _stream(stream))
    _check(st, "tardis_estimate_errors")
    return err, tot


def tardis_assign_thresholds(err, t: float, t_min: float, t_max: float, stream=None):
    """-> float32[n] thresholds: minimise sum err_i t_i with mean t and the given bounds."""
    out = torch.empty_like(err)
    _check(lib().tardis_assign_thresholds(_ptr(err), err.numel(), float(t), float(t_min), float(t_max), _ptr(out),
                                          _stream(stream)), "tardis_assign_thresholds")
    return out


class Layer:
    """Owner of a tardis_handle_t.  Keeps the borrowed weight tensors alive."""

    def __init__(self, handle, ffn: FFN, max_batch: int):
        self.handle, self.ffn, self.max_batch = handle, ffn, max_batch
        self.d, self.h = ffn.d, ffn.h
        self.torch_dtype = ffn.W1.dtype
        self.device = ffn.W1.device

    def close(self):
        if self.handle is not None:
            torch.cuda.synchronize()
            lib().tardis_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tardis_fold(ffn: FFN, lo, hi, a, c, max_batch: int = 1, sketch_bits: int = 8, deterministic: bool = False,
                margin: float = 0.0, folded_fp8: bool = False, stream=None) -> Layer:
    for t in (lo, hi, a, c):
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.float32 and t.numel() == ffn.h
    opts = tardis_fold_opts(sketch_bits, FP8_E4M3 if folded_fp8 else ffn.dtype, max_batch, 1 if deterministic else 0,
                            float(margin))
    handle = C.c_void_p()
    st = lib().tardis_fold(C.byref(ffn.desc), _ptr(lo), _ptr(hi), _ptr(a), _ptr(c), C.byref(opts),
                           _stream(stream), C.byref(handle))
    _check(st, "tardis_fold")
    return Layer(handle, ffn, max_batch)


def tardis_ffn_forward(L: Layer, x, y=None, stream=None):
    if y is None:
        y = torch.empty_like(x)
    _check(lib().tardis_ffn_forward(L.handle, _ptr(x), _ptr(y), _stream(stream)), "tardis_ffn_forward")
    return y


def tardis_ffn_forward_batched(L: Layer, x, y=None, stream=None):
    if y is None:
        y = torch.empty_like(x)
    _check(lib().tardis_ffn_forward_batched(L.handle, _ptr(x), x.shape[0], _ptr(y), _stream(stream)),
           "tardis_ffn_forward_batched")
    return y


def tardis_ffn_forward_static(L: Layer, x, y=None, mask_out=None, stream=None):
    """n <= 16 tokens with the library's static working memory (the call allocates nothing)."""
    if y is None:
        y = torch.empty_like(x)
    n = 1 if x.dim() == 1 else x.shape[0]
    _check(lib().tardis_ffn_forward_static(L.handle, _ptr(x), n, _ptr(y), _ptr(mask_out), _stream(stream)),
           "tardis_ffn_forward_static")
    return y


def tardis_stack_forward(layers, x, y=None, stream=None):
    """x: n x d through every layer in turn (RMS-normalised between layers)."""
    if y is None:
        y = torch.empty_like(x)
    arr = (C.c_void_p * len(layers))(*[L.handle for L in layers])
    n = 1 if x.dim() == 1 else x.shape[0]
    _check(lib().tardis_stack_forward(arr, len(layers), _ptr(x), n, _ptr(y), _stream(stream)), "tardis_stack_forward")
    return y


def tardis_set_next_layer(L: Layer, nxt):
    """Hint: `nxt` (a Layer or None) is the layer whose call follows L's."""
    _check(lib().tardis_set_next_layer(L.handle, nxt.handle if nxt is not None else None), "tardis_set_next_layer")


def tardis_dense_forward(L: Layer, x, y=None, stream=None):
    if y is None:
        y = torch.empty_like(x)
    n = 1 if x.dim() == 1 else x.shape[0]
    _check(lib().tardis_dense_forward(L.handle, _ptr(x), n, _ptr(y), _stream(stream)), "tardis_dense_forward")
    return y


def tardis_get_folded(L: Layer, stream=None):
    Wp = torch.empty(L.d, L.d, dtype=L.torch_dtype, device=L.device)
    bp = torch.empty(L.d, dtype=torch.float32, device=L.device)
    _check(lib().tardis_get_folded(L.handle, _ptr(Wp), _ptr(bp), _stream(stream)), "tardis_get_folded")
    return Wp, bp


def tardis_get_predictor_state(L: Layer, stream=None):
    Q = torch.empty(L.h, L.d, dtype=torch.int8, device=L.device)
    tlo = torch.empty(L.h, dtype=torch.float32, device=L.device)
    thi = torch.empty(L.h, dtype=torch.float32, device=L.device)
    _check(lib().tardis_get_predictor_state(L.handle, _ptr(Q), _ptr(tlo), _ptr(thi), _stream(stream)),
           "tardis_get_predictor_state")
    return Q, tlo, thi


def tardis_get_sketch_groups(L: Layer, stream=None):
    M = torch.empty(L.h, (L.d + 31) // 32, dtype=torch.uint8, device=L.device)
    _check(lib().tardis_get_sketch_groups(L.handle, _ptr(M), _stream(stream)), "tardis_get_sketch_groups")
    return M


def tardis_get_handover(L: Layer, n: int, stream=None):
    out = torch.empty(n, L.d, dtype=L.torch_dtype, device=L.device)
    _check(lib().tardis_get_handover(L.handle, n, _ptr(out), _stream(stream)), "tardis_get_handover")
    return out


def tardis_get_last_outliers(L: Layer, n: int, want_list: bool = True, stream=None):
    """-> (mask int32[n, ceil(h/32)] holding the uint32 words, counts int32[n], list int32[n, h] or None)."""
    words = (L.h + 31) // 32
    mask = torch.empty(n, words, dtype=torch.int32, device=L.device)
    counts = torch.empty(n, dtype=torch.int32, device=L.device)
    lst = torch.empty(n, L.h, dtype=torch.int32, device=L.device) if want_list else None
    _check(lib().tardis_get_last_outliers(L.handle, n, _ptr(mask), _ptr(counts), _ptr(lst), _stream(stream)),
           "tardis_get_last_outliers")
    return mask, counts, lst


def tardis_get_last_union(L: Layer, n: int, want_mask: bool = False, stream=None):
    """-> (union_count int32[1] on the device, union mask int32[ceil(h/32)] or None)."""
    cnt = torch.empty(1, dtype=torch.int32, device=L.device)
    um = torch.empty((L.h + 31) // 32, dtype=torch.int32, device=L.device) if want_mask else None
    _check(lib().tardis_get_last_union(L.handle, n, _ptr(um), _ptr(cnt), _stream(stream)), "tardis_get_last_union")
    return cnt, um


def tardis_release_memory():
    """Returns to the device the memory that the library keeps of the layer closed last (see tardis_destroy)."""
    _check(lib().tardis_release_memory(), "tardis_release_memory")


@functools.lru_cache(maxsize=4096)
def _linear_work_bytes(sizes, experts, x_rows, pitch, ordered, rows, x_at, W_at):
    """Of a call of these sizes (n_in, n_out, dtype, out_dtype, act) with operands at addresses of these remainders by 16."""
    bytes_ = C.c_int64()
    desc = tardis_linear_desc(*sizes, 0, 256 + W_at, None)
    if experts:
        _check(lib().tardis_grouped_linear_workspace(desc, experts, 256 + x_at, x_rows, pitch, ordered, rows, bytes_), "tardis_grouped_linear_workspace")
    else:
        _check(lib().tardis_linear_workspace(desc, 256 + x_at, rows, pitch, bytes_), "tardis_linear_workspace")
    return bytes_.value


@functools.lru_cache(maxsize=1024)
def _route_work_bytes(n, experts, k):
    bytes_ = C.c_int64()
    _check(lib().tardis_moe_route_workspace(n, experts, k, bytes_), "tardis_moe_route_workspace")
    return bytes_.value


def _on(stream):
    """The stream that a call is given, as the current one: outputs and working memory then are its own, and not given to other work while it runs."""
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream())


def _empty(n, width, dtype, device):
    return torch.empty_strided((n, width), (width, 1), dtype=dtype, device=device)   # (half the host time of torch.empty)


def _rows(x, n_in):
    """Rows that may lie further apart than they are long -> their number and distance."""
    assert x.is_cuda and x.dim() == 2 and x.shape[1] == n_in
    n, (pitch, step) = x.shape[0], x.stride()
    assert (step == 1 or n_in == 1) and (pitch >= n_in or n <= 1)
    return n, pitch if n > 1 else n_in


def tardis_linear(x, W, b=None, act: str = "identity", residual=None, out_dtype=None, y=None, stream=None):
    """-> n x n_out: act(x W^T + b) + residual.  Rows of x may have a pitch; out_dtype: of residual and y (default: x's)."""
    if stream is not None:
        with _on(stream):
            return tardis_linear(x, W, b, act, residual, out_dtype, y)
    n_out, n_in = W.shape
    n, pitch = _rows(x, n_in)
    dt, dev = x.dtype, x.get_device()
    out_dtype = out_dtype or dt
    assert W.is_contiguous() and W.dtype == dt and W.get_device() == dev
    assert b is None or (b.is_contiguous() and b.dtype == dt and b.numel() == n_out and b.get_device() == dev)
    assert residual is None or (residual.is_contiguous() and residual.dtype == out_dtype and residual.shape == (n, n_out) and residual.get_device() == dev)
    if y is None:
        y = _empty(n, n_out, out_dtype, x.device)
    else:
        assert y.is_contiguous() and y.dtype == out_dtype and y.shape == (n, n_out) and y.get_device() == dev
    sizes, x_at, W_at = (n_in, n_out, _DTYPE_CODE[dt], _DTYPE_CODE[out_dtype], ACT[act]), x.data_ptr(), W.data_ptr()
    desc = tardis_linear_desc(*sizes, 0, W_at, None if b is None else b.data_ptr())
    bytes_ = _linear_work_bytes(sizes, 0, n, pitch, 0, n, x_at & 15, W_at & 15)
    work = torch.empty(bytes_, dtype=torch.uint8, device=x.device) if bytes_ else None
    _check(lib().tardis_linear(desc, x_at, n, pitch, _ptr(residual), y.data_ptr(), _ptr(work), bytes_, _stream(None)), "tardis_linear")
    return y


def tardis_grouped_linear(x, W, offsets, b=None, act: str = "identity", order=None, per_token: int = 1, out_dtype=None, y=None, stream=None):
    """-> positions x n_out: act(x[order[p] // per_token] W[e]^T + b[e]) at positions offsets[e] <= p < offsets[e + 1]; without
    an order x[p].  W: experts x n_out x n_in.  Rows of y in no group are not written."""
    if stream is not None:
        with _on(stream):
            return tardis_grouped_linear(x, W, offsets, b, act, order, per_token, out_dtype, y)
    experts, n_out, n_in = W.shape
    x_rows, pitch = _rows(x, n_in)
    dt, dev = x.dtype, x.get_device()
    out_dtype = out_dtype or dt
    assert W.is_contiguous() and W.dtype == dt and W.get_device() == dev
    assert b is None or (b.is_contiguous() and b.dtype == dt and b.numel() == experts * n_out and b.get_device() == dev)
    assert offsets.is_contiguous() and offsets.dtype == torch.int32 and offsets.numel() == experts + 1 and offsets.get_device() == dev
    assert order is None or (order.is_contiguous() and order.dtype == torch.int32 and order.get_device() == dev)
    positions = x_rows if order is None else order.numel()
    if y is None:
        y = _empty(positions, n_out, out_dtype, x.device)
    else:
        assert y.is_contiguous() and y.dtype == out_dtype and y.shape == (positions, n_out) and y.get_device() == dev
    sizes, x_at, W_at, ordered = (n_in, n_out, _DTYPE_CODE[dt], _DTYPE_CODE[out_dtype], ACT[act]), x.data_ptr(), W.data_ptr(), order is not None
    desc = tardis_linear_desc(*sizes, 0, W_at, None if b is None else b.data_ptr())
    bytes_ = _linear_work_bytes(sizes, experts, x_rows, pitch, int(ordered), positions, x_at & 15, W_at & 15)
    work = torch.empty(bytes_, dtype=torch.uint8, device=x.device) if bytes_ else None
    _check(lib().tardis_grouped_linear(desc, experts, x_at, x_rows, pitch, offsets.data_ptr(), _ptr(order), per_token, positions, y.data_ptr(),
                                       _ptr(work), bytes_, _stream(None)), "tardis_grouped_linear")
    return y


def tardis_moe_route(logits, k: int, renormalise: bool = True, stream=None):
    """logits n x experts -> (ids int32[n, k], weights float32[n, k], offsets int32[experts + 1], order int32[n k], place int32[n, k])."""
    if stream is not None:
        with _on(stream):
            return tardis_moe_route(logits, k, renormalise)
    n, experts = logits.shape
    assert logits.is_cuda and logits.is_contiguous()
    dev = logits.device
    ids, place, weights = _empty(n, k, torch.int32, dev), _empty(n, k, torch.int32, dev), _empty(n, k, torch.float32, dev)
    order = torch.empty_strided((n * k,), (1,), dtype=torch.int32, device=dev)
    offsets = torch.empty_strided((experts + 1,), (1,), dtype=torch.int32, device=dev)
    bytes_ = _route_work_bytes(n, experts, k)
    work = torch.empty(bytes_, dtype=torch.uint8, device=dev) if bytes_ else None
    _check(lib().tardis_moe_route(logits.data_ptr(), n, experts, k, _DTYPE_CODE[logits.dtype], 1 if renormalise else 0, ids.data_ptr(), weights.data_ptr(),
                                  offsets.data_ptr(), order.data_ptr(), place.data_ptr(), _ptr(work), bytes_, _stream(None)), "tardis_moe_route")
    return ids, weights, offsets, order, place


def tardis_moe_combine(z, place, weights, residual=None, out_dtype=None, y=None, stream=None):
    """-> n x d: residual[t] + sum_j weights[t, j] z[place[t, j]]; a place below 0 is a dropped slot.  out_dtype: of residual and y (default: z's)."""
    if stream is not None:
        with _on(stream):
            return tardis_moe_combine(z, place, weights, residual, out_dtype, y)
    (rows, d), (n, k), dev = z.shape, place.shape, z.get_device()
    out_dtype = out_dtype or z.dtype
    assert z.is_cuda and z.is_contiguous() and place.is_contiguous() and place.dtype == torch.int32 and place.get_device() == dev
    assert weights.is_contiguous() and weights.dtype == torch.float32 and weights.shape == (n, k) and weights.get_device() == dev
    assert residual is None or (residual.is_contiguous() and residual.dtype == out_dtype and residual.shape == (n, d) and residual.get_device() == dev)
    if y is None:
        y = _empty(n, d, out_dtype, z.device)
    else:
        assert y.is_contiguous() and y.dtype == out_dtype and y.shape == (n, d) and y.get_device() == dev
    _check(lib().tardis_moe_combine(z.data_ptr(), rows, place.data_ptr(), weights.data_ptr(), n, k, d, _DTYPE_CODE[z.dtype], _ptr(residual), y.data_ptr(),
                                    _DTYPE_CODE[out_dtype], _stream(None)), "tardis_moe_combine")
    return y


# ---------------------------------------------------------------- norms, layers in 8 and 4 bits
FP8 = torch.float8_e4m3fn
FP8_EXACT = 0x100                  # tardis.h's TARDIS_FP8_EXACT


def _at(t):
    """Where a tensor is (None: nowhere)"""
    return None if t is None else t.data_ptr()


def _empty1(n, dtype, device):
    return torch.empty_strided((n,), (1,), dtype=dtype, device=device)


_OUT_CODE = {torch.float32: F32, torch.bfloat16: BF16, FP8: FP8_E4M3}


def tardis_rms_norm(x, weight=None, residual=None, eps: float = 1e-6, out_dtype=None, sum=None, y=None, scales=None, stream=None):
    """s = x + residual -> y = s / sqrt(mean(s^2) + eps) * weight, in out_dtype (default: x's; torch.float8_e4m3fn: codes, with a scale for each row).

    Returns y; (y, scales) with codes; with a residual s behind them: (y, sum), (y, scales, sum).  Rows of x may have a pitch.  sum, y, scales:
    where to write them (sum may be the residual itself)."""
    if stream is not None:
        with _on(stream):
            return tardis_rms_norm(x, weight, residual, eps, out_dtype, sum, y, scales)
    d = x.shape[-1]
    n, pitch = _rows(x, d)
    dt, device, dev = x.dtype, x.device, x.get_device()
    if out_dtype is None:
        out_dtype = dt
    codes = out_dtype == FP8
    assert weight is None or (weight.is_contiguous() and weight.dtype == dt and weight.numel() == d and weight.get_device() == dev)
    if residual is not None:
        assert residual.is_contiguous() and residual.dtype == dt and residual.shape == (n, d) and residual.get_device() == dev
        if sum is None:
            sum = _empty(n, d, dt, device)
    assert sum is None or (sum.is_contiguous() and sum.dtype == dt and sum.shape == (n, d) and sum.get_device() == dev)
    if y is None:
        y = _empty(n, d, out_dtype, device)
    else:
        assert y.is_contiguous() and y.dtype == out_dtype and y.shape == (n, d) and y.get_device() == dev
    if codes and scales is None:
        scales = _empty1(n, torch.float32, device)
    else:
        assert scales is None or (codes and scales.is_contiguous() and scales.dtype == torch.float32 and scales.shape == (n,) and scales.get_device() == dev)
    desc = tardis_norm_desc(d, _DTYPE_CODE[dt], _OUT_CODE[out_dtype], eps, 0, _at(weight))
    _check(lib().tardis_rms_norm(desc, x.data_ptr(), n, pitch, _at(residual), _at(sum), y.data_ptr(), _at(scales), _stream(None)), "tardis_rms_norm")
    if codes:
        return (y, scales) if residual is None else (y, scales, sum)
    return y if residual is None else (y, sum)


def tardis_fp8_rows(x, codes=None, scales=None, stream=None):
    """n x d -> (e4m3 codes n x d, scales float32[n]): a row is its codes times its scale.  Rows of x may have a pitch."""
    if stream is not None:
        with _on(stream):
            return tardis_fp8_rows(x, codes, scales)
    d = x.shape[-1]
    n, pitch = _rows(x, d)
    dev = x.get_device()
    if codes is None:
        codes = _empty(n, d, FP8, x.device)
    else:
        assert codes.is_contiguous() and codes.dtype == FP8 and codes.shape == (n, d) and codes.get_device() == dev
    if scales is None:
        scales = _empty1(n, torch.float32, x.device)
    else:
        assert scales.is_contiguous() and scales.dtype == torch.float32 and scales.shape == (n,) and scales.get_device() == dev
    _check(lib().tardis_fp8_rows(x.data_ptr(), n, d, pitch, _DTYPE_CODE[x.dtype], codes.data_ptr(), scales.data_ptr(), _stream(None)), "tardis_fp8_rows")
    return codes, scales


@functools.lru_cache(maxsize=4096)
def _fp8_work_bytes(n_in, n_out, out, act, n, pitch, x_at, W_at):
    bytes_ = C.c_int64()
    _check(lib().tardis_linear_fp8_workspace(tardis_linear_fp8_desc(n_in, n_out, out, act, 256 + W_at, None, None), 256 + x_at, n, pitch, bytes_),
           "tardis_linear_fp8_workspace")
    return bytes_.value


@functools.lru_cache(maxsize=4096)
def _four_work_bytes(n_in, n_out, dtype, out, act, group, n, pitch):
    bytes_ = C.c_int64()
    _check(lib().tardis_linear_4bit_workspace(tardis_linear_4bit_desc(n_in, n_out, dtype, out, act, group, 256, 256, None, None), n, pitch, bytes_),
           "tardis_linear_4bit_workspace")
    return bytes_.value


def _layer_outputs(n, n_out, out_dtype, b, residual, y, x):
    """The checks that layers in 8 and 4 bits share -> y"""
    dev = x.get_device()
    assert b is None or (b.is_contiguous() and b.dtype == out_dtype and b.numel() == n_out and b.get_device() == dev)
    assert residual is None or (residual.is_contiguous() and residual.dtype == out_dtype and residual.shape == (n, n_out) and residual.get_device() == dev)
    if y is None:
        return _empty(n, n_out, out_dtype, x.device)
    assert y.is_contiguous() and y.dtype == out_dtype and y.shape == (n, n_out) and y.get_device() == dev
    return y


def tardis_linear_fp8(x, x_scales, W, W_scales, b=None, act: str = "identity", residual=None, out_dtype=torch.bfloat16, y=None, stream=None,
                      exact: bool = False):
    """-> n x n_out: act(x W^T + b) + residual with x and W in e4m3, each row with a scale (None: ones).  Rows of x may have a pitch; out_dtype: of b,
    residual and y.  exact: sums of exact products also for outputs in bf16, which by default lose up to 2^-10 sum |x W| (tardis.h)."""
    if stream is not None:
        with _on(stream):
            return tardis_linear_fp8(x, x_scales, W, W_scales, b, act, residual, out_dtype, y, exact=exact)
    n_out, n_in = W.shape
    n, pitch = _rows(x, n_in)
    dev = x.get_device()
    assert W.is_contiguous() and W.dtype == FP8 and x.dtype == FP8 and W.get_device() == dev
    assert x_scales is None or (x_scales.is_contiguous() and x_scales.dtype == torch.float32 and x_scales.numel() == n and x_scales.get_device() == dev)
    assert W_scales is None or (W_scales.is_contiguous() and W_scales.dtype == torch.float32 and W_scales.numel() == n_out and W_scales.get_device() == dev)
    y = _layer_outputs(n, n_out, out_dtype, b, residual, y, x)
    out, a, x_at, W_at = _DTYPE_CODE[out_dtype], ACT[act] | (FP8_EXACT if exact else 0), x.data_ptr(), W.data_ptr()
    desc = tardis_linear_fp8_desc(n_in, n_out, out, a, W_at, _at(W_scales), _at(b))
    bytes_ = _fp8_work_bytes(n_in, n_out, out, a, n, pitch, x_at & 15, W_at & 15)
    work = torch.empty(bytes_, dtype=torch.uint8, device=x.device) if bytes_ else None
    _check(lib().tardis_linear_fp8(desc, x_at, _at(x_scales), n, pitch, _at(residual), y.data_ptr(), _at(work), bytes_, _stream(None)), "tardis_linear_fp8")
    return y


def tardis_pack_4bit(codes, group: int):
    """Codes n_out x n_in, 0 to 15 -> what tardis_linear_4bit reads: int32[n_out, G group / 8], G = ceil(n_in / group), on the codes' device (rows
    are filled with zeros to whole groups).  Done once for a layer, in torch."""
    n_out, n_in = codes.shape
    words = torch.zeros(n_out, -(-n_in // group) * group, dtype=torch.int64, device=codes.device)
    words[:, :n_in] = codes
    at = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], device=codes.device)
    words = ((words.view(n_out, -1, 8) & 15) << at).sum(2)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def tardis_linear_4bit(x, W, scales, zeros=None, b=None, group: int = 128, act: str = "identity", residual=None, out_dtype=None, y=None, stream=None):
    """-> n x n_out: act(x W'^T + b) + residual, W' = scales (codes - zeros) for each group of columns.  W: tardis_pack_4bit's; scales: n_out x G,
    dtype of x; zeros: uint8 n_out x G (None: 8).  Rows of x may have a pitch; out_dtype: of b, residual and y (default: x's)."""
    if stream is not None:
        with _on(stream):
            return tardis_linear_4bit(x, W, scales, zeros, b, group, act, residual, out_dtype, y)
    n_out, n_in = W.shape[0], x.shape[-1]
    n, pitch = _rows(x, n_in)
    dt, dev = x.dtype, x.get_device()
    out_dtype = out_dtype or dt
    assert group in (32, 64, 128)
    groups = -(-n_in // group)
    assert W.is_contiguous() and W.dtype == torch.int32 and W.shape == (n_out, groups * group // 8) and W.get_device() == dev
    assert scales.is_contiguous() and scales.dtype == dt and scales.shape == (n_out, groups) and scales.get_device() == dev
    assert zeros is None or (zeros.is_contiguous() and zeros.dtype == torch.uint8 and zeros.shape == (n_out, groups) and zeros.get_device() == dev)
    y = _layer_outputs(n, n_out, out_dtype, b, residual, y, x)
    sizes = (n_in, n_out, _DTYPE_CODE[dt], _DTYPE_CODE[out_dtype], ACT[act], group)
    desc = tardis_linear_4bit_desc(*sizes, W.data_ptr(), scales.data_ptr(), _at(zeros), _at(b))
    bytes_ = _four_work_bytes(*sizes, n, pitch)
    work = torch.empty(bytes_, dtype=torch.uint8, device=x.device) if bytes_ else None
    _check(lib().tardis_linear_4bit(desc, x.data_ptr(), n, pitch, _at(residual), y.data_ptr(), _at(work), bytes_, _stream(None)), "tardis_linear_4bit")
    return y
