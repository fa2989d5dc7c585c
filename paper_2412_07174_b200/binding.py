"""Binding of libscap_b200.so: same names as the C ABI, marshalling only.

The decode calls go through a small native helper (csrc/scap_pycall.c), the others through ctypes: at one token the host
bounds a call, and marshalling was most of it (scap_sparse_fc, K = N = 1024, one row: 10.5 -> 5.3 us a call, 4.1 us on the device)."""
from __future__ import annotations

import ctypes as C
import os
import warnings

import torch

__all__ = [
    "SCAP_F16", "SCAP_BF16", "SCAP_F32", "ScapError", "lib", "lib_path", "status_string", "scap_version", "scap_tune", "scap_device_status",
    "scap_calibrate_workspace", "scap_calibrate", "scap_calibrate_ex", "SCAP_MODE_HISTOGRAM", "SCAP_MODE_MEAN", "SCAP_MODE_MEDIAN", "SCAP_MODE_KDE",
    "SCAP_ETA_PER_CHANNEL", "SCAP_ETA_SCALAR", "scap_fold_bias_workspace", "scap_fold_bias",
    "scap_fc_workspace", "scap_sparse_fc", "scap_dense_fc", "scap_sparse_fc_q8", "scap_dense_fc_q8", "scap_fold_bias_q8",
    "scap_sparse_fc_q4", "scap_dense_fc_q4", "scap_fold_bias_q4", "scap_grouped_workspace", "scap_sparse_fc_grouped",
    "scap_fc_host_workspace", "scap_sparse_fc_host",
    "scap_glu_workspace", "scap_glu_ffn", "scap_gelu_ffn_workspace", "scap_gelu_ffn", "scap_glu_static_capacity", "scap_glu_ffn_static", "scap_moe_workspace",
    "scap_moe_ffn", "ScapExpert", "dtype_of", "EXPORTS",
    "SCAP_ACT_NONE", "SCAP_ACT_RELU", "SCAP_ACT_SILU", "SCAP_ACT_GELU", "SCAP_ACT_GELU_TANH", "scap_fc_act_workspace", "scap_fc_act",
    "ScapKv4", "scap_kv4_page_bytes", "scap_kv4_append", "scap_kv4_read", "scap_kv4_attend_workspace", "scap_kv4_attend",
    "scap_kv4_pages_workspace", "scap_kv4_copy", "scap_kv4_fork", "scap_kv4_free", "scap_kv4_reserve", "scap_kv4_compact",
]

SCAP_F16, SCAP_BF16, SCAP_F32 = 0, 1, 2
SCAP_ACT_NONE, SCAP_ACT_RELU, SCAP_ACT_SILU, SCAP_ACT_GELU, SCAP_ACT_GELU_TANH = range(5)
_HERE = os.path.dirname(os.path.abspath(__file__))

# every symbol include/scap.h declares
EXPORTS = [
    "scap_status_string", "scap_version", "scap_tune", "scap_device_status", "scap_calibrate_workspace", "scap_calibrate",
    "scap_calibrate_ex", "scap_fold_bias_workspace", "scap_fold_bias", "scap_fc_workspace", "scap_sparse_fc", "scap_dense_fc",
    "scap_sparse_fc_q8", "scap_dense_fc_q8", "scap_fold_bias_q8", "scap_sparse_fc_q4", "scap_dense_fc_q4", "scap_fold_bias_q4",
    "scap_grouped_workspace", "scap_sparse_fc_grouped", "scap_fc_host_workspace", "scap_sparse_fc_host", "scap_glu_workspace", "scap_glu_ffn", "scap_gelu_ffn_workspace",
    "scap_gelu_ffn", "scap_glu_static_capacity", "scap_glu_ffn_static", "scap_moe_workspace", "scap_moe_ffn",
    "scap_fc_act_workspace", "scap_fc_act", "scap_kv4_page_bytes", "scap_kv4_append", "scap_kv4_read", "scap_kv4_attend_workspace", "scap_kv4_attend",
    "scap_kv4_pages_workspace", "scap_kv4_copy", "scap_kv4_fork", "scap_kv4_free", "scap_kv4_reserve", "scap_kv4_compact",
]


class ScapError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s" % (where, status_string(code)))


class ScapExpert(C.Structure):
    """Mirror of ``scap_expert``: device pointers of one expert's weights and calibration."""
    _fields_ = [(n, C.c_void_p) for n in ("Wgu", "Wd", "m1", "tau1", "bgu_fused", "m2", "tau2", "bd_fused")]


def lib_path() -> str:
    return os.path.join(_HERE, "libscap_b200.so")


_lib = None
_call = None    # call(entry, arg, ...) -> status: the native helper, or ctypes where it is not built
_call_real = None  # call_real(entry, x, arg, ...) -> status, for an entry point with one double: the native helper only
_entry = {}     # name -> what `_call` takes as the entry point: its address, or the ctypes function


def lib():
    """Loads the CUDA library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError("%s is missing: run `python -m paper_2412_07174_b200.build` (needs nvcc)" % path)
    L = C.CDLL(path)
    vp, i, sz, d = C.c_void_p, C.c_int, C.c_size_t, C.c_double
    L.scap_status_string.argtypes = [i]
    L.scap_status_string.restype = C.c_char_p
    L.scap_version.argtypes = []
    L.scap_version.restype = i
    L.scap_tune.argtypes = [C.c_char_p, i]
    L.scap_tune.restype = i
    L.scap_device_status.argtypes = []
    L.scap_device_status.restype = i
    L.scap_calibrate_workspace.argtypes = [i, i, i]
    L.scap_calibrate_workspace.restype = sz
    L.scap_calibrate.argtypes = [vp, i, i, i, d, i, vp, vp, vp, sz, vp]
    L.scap_calibrate.restype = i
    L.scap_calibrate_ex.argtypes = [vp, i, i, i, d, i, i, i, vp, vp, vp, sz, vp]
    L.scap_calibrate_ex.restype = i
    L.scap_fold_bias_workspace.argtypes = [i, i]
    L.scap_fold_bias_workspace.restype = sz
    L.scap_fold_bias.argtypes = [vp, vp, vp, i, i, i, vp, vp, sz, vp]
    L.scap_fold_bias.restype = i
    L.scap_fc_workspace.argtypes = [i, i, i]
    L.scap_fc_workspace.restype = sz
    L.scap_sparse_fc.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp, vp, vp, sz, vp]
    L.scap_sparse_fc.restype = i
    L.scap_dense_fc.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.scap_dense_fc.restype = i
    L.scap_sparse_fc_q8.argtypes = [vp, i, vp, vp, vp, vp, vp, vp, i, i, i, vp, vp, vp, sz, vp]
    L.scap_sparse_fc_q8.restype = i
    L.scap_dense_fc_q8.argtypes = [vp, i, vp, vp, vp, vp, i, i, i, vp, sz, vp]
    L.scap_dense_fc_q8.restype = i
    L.scap_fold_bias_q8.argtypes = [vp, vp, vp, vp, i, i, vp, vp, sz, vp]
    L.scap_fold_bias_q8.restype = i
    L.scap_sparse_fc_q4.argtypes = [vp, i, vp, vp, vp, i, vp, vp, vp, vp, i, i, i, vp, vp, vp, sz, vp]
    L.scap_sparse_fc_q4.restype = i
    L.scap_dense_fc_q4.argtypes = [vp, i, vp, vp, vp, i, vp, vp, i, i, i, vp, sz, vp]
    L.scap_dense_fc_q4.restype = i
    L.scap_fold_bias_q4.argtypes = [vp, vp, vp, i, vp, vp, i, i, vp, vp, sz, vp]
    L.scap_fold_bias_q4.restype = i
    L.scap_grouped_workspace.argtypes = []
    L.scap_grouped_workspace.restype = sz
    L.scap_sparse_fc_grouped.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp, vp, sz, vp]
    L.scap_sparse_fc_grouped.restype = i
    L.scap_fc_host_workspace.argtypes = [i, i, i]
    L.scap_fc_host_workspace.restype = sz
    L.scap_sparse_fc_host.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.scap_sparse_fc_host.restype = i
    L.scap_glu_workspace.argtypes = [i, i, i]
    L.scap_glu_workspace.restype = sz
    L.scap_glu_ffn.argtypes = [vp] * 10 + [i, i, i, i] + [vp] * 5 + [vp, sz, vp]
    L.scap_glu_ffn.restype = i
    L.scap_gelu_ffn_workspace.argtypes = [i, i, i]
    L.scap_gelu_ffn_workspace.restype = sz
    L.scap_gelu_ffn.argtypes = [vp] * 10 + [i, i, i, i] + [vp] * 5 + [vp, sz, vp]
    L.scap_gelu_ffn.restype = i
    L.scap_glu_static_capacity.argtypes = []
    L.scap_glu_static_capacity.restype = sz
    L.scap_glu_ffn_static.argtypes = [vp] * 10 + [i, i, i, i] + [vp, vp]
    L.scap_glu_ffn_static.restype = i
    L.scap_moe_workspace.argtypes = [i, i, i, i, i]
    L.scap_moe_workspace.restype = sz
    L.scap_moe_ffn.argtypes = [vp, vp, C.POINTER(ScapExpert), i, i, vp, i, i, i, i, vp, vp, vp, sz, vp]
    L.scap_moe_ffn.restype = i
    i64 = C.c_int64
    L.scap_fc_act_workspace.argtypes = [i, i, i, i64]
    L.scap_fc_act_workspace.restype = sz
    L.scap_fc_act.argtypes = [vp, i64, vp, vp, i, vp, i64, vp, i64, i, i, i, i, i, vp, sz, vp]
    L.scap_fc_act.restype = i
    L.scap_kv4_page_bytes.argtypes = [i, i, i, i]
    L.scap_kv4_page_bytes.restype = sz
    for n in ("scap_kv4_append", "scap_kv4_read"):
        getattr(L, n).argtypes = [vp, vp, i64, vp, i64, vp, i, i, vp]
        getattr(L, n).restype = i
    L.scap_kv4_attend_workspace.argtypes = [i, i, i, i, i]
    L.scap_kv4_attend_workspace.restype = sz
    L.scap_kv4_attend.argtypes = [vp, vp, i64, vp, i64, vp, i, i, d, i, i, vp, sz, vp]
    L.scap_kv4_attend.restype = i
    L.scap_kv4_pages_workspace.argtypes = [i, i]
    L.scap_kv4_pages_workspace.restype = sz
    for n, a in (("copy", [vp, vp, vp, i, vp]), ("fork", [vp, vp, vp, i, vp, vp, sz, vp]), ("free", [vp, vp, i, vp]), ("reserve", [vp, vp, vp, vp, sz, vp]), ("compact", [vp, vp, vp, sz, vp])):
        getattr(L, "scap_kv4_" + n).argtypes = a
        getattr(L, "scap_kv4_" + n).restype = i
    global _call, _call_real
    try:
        from ._scap_call import call, call_real
        _entry.update({n: C.cast(getattr(L, n), C.c_void_p).value for n in EXPORTS})
    except ImportError as e:
        warnings.warn("%s: calls go through ctypes, about 5 us slower each; `python -m paper_2412_07174_b200.build` builds the helper" % e)
        call, call_real = _ctypes_call, None
        _entry.update({n: getattr(L, n) for n in EXPORTS})
    _call, _call_real = call, call_real
    _lib = L
    return L


def _ctypes_call(entry, *args) -> int:
    """What the native helper does, by ctypes."""
    return entry(*[a if isinstance(a, C.c_double) else _ptr(a) for a in args])


def _invoke(name: str, *args) -> None:
    """Calls the entry point `name`; an argument is a tensor (its address), an address, an integer or None."""
    if _lib is None:
        lib()
    code = _call(_entry[name], *args)
    if code != 0:
        raise ScapError(code, name)


def _invoke_real(name: str, x: float, at: int, *args) -> None:
    """The same for an entry point that has one double, `x`, before its argument number `at`."""
    if _lib is None:
        lib()
    if _call_real is not None and _call is not _ctypes_call:
        code = _call_real(_entry[name], x, *args)
    else:
        code = _ctypes_call(getattr(_lib, name), *args[:at], C.c_double(x), *args[at:])
    if code != 0:
        raise ScapError(code, name)


def status_string(code: int) -> str:
    return lib().scap_status_string(int(code)).decode()


def scap_version() -> int:
    return lib().scap_version()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise ScapError(code, where)


def scap_tune(key: str, value: int) -> None:
    _check(lib().scap_tune(key.encode(), int(value)), "scap_tune")


def scap_device_status() -> None:
    """Synchronises the device; raises ScapError(SCAP_ERR_TIMEOUT) if a bounded wait of the tcgen05 kernel ran out."""
    _check(lib().scap_device_status(), "scap_device_status")


def _ptr(t):
    """Address of a tensor's storage, an int address, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        if torch.cuda.is_initialized():  # the current stream of the current device, without a Stream object
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_DTYPES = {torch.float16: SCAP_F16, torch.bfloat16: SCAP_BF16}


def dtype_of(t: torch.Tensor) -> int:
    code = _DTYPES.get(t.dtype)
    if code is not None:
        return code
    raise TypeError("weights/activations must be float16 or bfloat16, got %s" % t.dtype)


def _ws(ws):
    return (ws.data_ptr(), ws.nbytes) if ws is not None else (None, 0)


def scap_calibrate_workspace(T: int, K: int, nbins: int) -> int:
    return lib().scap_calibrate_workspace(T, K, nbins)


def scap_calibrate(x_calib, sparsity: float, nbins: int, m_out, tau_out, ws, stream=None) -> None:
    T, K = x_calib.shape
    p, n = _ws(ws)
    _check(lib().scap_calibrate(_ptr(x_calib), T, K, dtype_of(x_calib), float(sparsity), nbins, _ptr(m_out), _ptr(tau_out),
                                p, n, _stream(stream)), "scap_calibrate")


SCAP_MODE_HISTOGRAM, SCAP_MODE_MEAN, SCAP_MODE_MEDIAN, SCAP_MODE_KDE = 0, 1, 2, 3
SCAP_ETA_PER_CHANNEL, SCAP_ETA_SCALAR = 0, 1


def scap_calibrate_ex(x_calib, sparsity: float, estimator: int, scope: int, nbins: int, m_out, tau_out, ws, stream=None) -> None:
    T, K = x_calib.shape
    p, n = _ws(ws)
    _check(lib().scap_calibrate_ex(_ptr(x_calib), T, K, dtype_of(x_calib), float(sparsity), int(estimator), int(scope), nbins,
                                   _ptr(m_out), _ptr(tau_out), p, n, _stream(stream)), "scap_calibrate_ex")


def scap_fold_bias_workspace(K: int, N: int) -> int:
    return lib().scap_fold_bias_workspace(K, N)


def scap_fold_bias(W, m, b, b_fused, ws, stream=None) -> None:
    K, N = W.shape
    p, n = _ws(ws)
    _check(lib().scap_fold_bias(_ptr(W), _ptr(m), _ptr(b), K, N, dtype_of(W), _ptr(b_fused), p, n, _stream(stream)),
           "scap_fold_bias")


def scap_fc_workspace(B: int, K: int, N: int) -> int:
    return lib().scap_fc_workspace(B, K, N)


def scap_sparse_fc(x, W, m, tau, b_fused, y, ws, idx_out=None, nnz_out=None, stream=None) -> None:
    B, K = x.shape
    N = W.shape[1]
    p, n = _ws(ws)
    _invoke("scap_sparse_fc", x, W, m, tau, b_fused, y, B, K, N, dtype_of(W), idx_out, nnz_out, p, n, _stream(stream))


def scap_dense_fc(x, W, b, y, ws, stream=None) -> None:
    B, K = x.shape
    N = W.shape[1]
    p, n = _ws(ws)
    _invoke("scap_dense_fc", x, W, b, y, B, K, N, dtype_of(W), p, n, _stream(stream))


def scap_sparse_fc_q8(x, Wq, wscale, m, tau, b_fused, y, ws, idx_out=None, nnz_out=None, stream=None) -> None:
    """Sparse FC on 8-bit weights: Wq int8 [K, N], wscale fp32 [K] (one scale per input channel)."""
    B, K = x.shape
    N = Wq.shape[1]
    p, n = _ws(ws)
    _invoke("scap_sparse_fc_q8", x, dtype_of(x), Wq, wscale, m, tau, b_fused, y, B, K, N, idx_out, nnz_out, p, n, _stream(stream))


def scap_dense_fc_q8(x, Wq, wscale, b, y, ws, stream=None) -> None:
    B, K = x.shape
    N = Wq.shape[1]
    p, n = _ws(ws)
    _invoke("scap_dense_fc_q8", x, dtype_of(x), Wq, wscale, b, y, B, K, N, p, n, _stream(stream))


def scap_fold_bias_q8(Wq, wscale, m, b, b_fused, ws, stream=None) -> None:
    K, N = Wq.shape
    p, n = _ws(ws)
    _check(lib().scap_fold_bias_q8(_ptr(Wq), _ptr(wscale), _ptr(m), _ptr(b), K, N, _ptr(b_fused), p, n, _stream(stream)),
           "scap_fold_bias_q8")


def scap_sparse_fc_q4(x, Wq, scale, zero, group, m, tau, b_fused, y, ws, idx_out=None, nnz_out=None, stream=None) -> None:
    """Sparse FC on group-wise 4-bit weights: Wq uint8 [K, N/2] (two codes per byte), scale fp32 and zero uint8 [K/group, N]."""
    B, K = x.shape
    N = Wq.shape[1] * 2
    p, n = _ws(ws)
    _invoke("scap_sparse_fc_q4", x, dtype_of(x), Wq, scale, zero, int(group), m, tau, b_fused, y, B, K, N, idx_out, nnz_out, p, n,
            _stream(stream))


def scap_dense_fc_q4(x, Wq, scale, zero, group, b, y, ws, stream=None) -> None:
    B, K = x.shape
    N = Wq.shape[1] * 2
    p, n = _ws(ws)
    _invoke("scap_dense_fc_q4", x, dtype_of(x), Wq, scale, zero, int(group), b, y, B, K, N, p, n, _stream(stream))


def scap_fold_bias_q4(Wq, scale, zero, group, m, b, b_fused, ws, stream=None) -> None:
    K, N = Wq.shape[0], Wq.shape[1] * 2
    p, n = _ws(ws)
    _check(lib().scap_fold_bias_q4(_ptr(Wq), _ptr(scale), _ptr(zero), int(group), _ptr(m), _ptr(b), K, N, _ptr(b_fused), p, n,
                                   _stream(stream)), "scap_fold_bias_q4")


def scap_grouped_workspace() -> int:
    return lib().scap_grouped_workspace()


def scap_sparse_fc_grouped(x, W, m, tau, b_fused, y, groups, ws, stream=None) -> None:
    """Sparse FC with one union mask per group of rows; ``groups`` is a host sequence of B group numbers 0..15."""
    B, K = x.shape
    N = W.shape[1]
    p, n = _ws(ws)
    arr = (C.c_int * B)(*[int(g) for g in groups])
    _invoke("scap_sparse_fc_grouped", x, W, m, tau, b_fused, y, B, K, N, dtype_of(W), C.addressof(arr), p, n, _stream(stream))


def scap_fc_host_workspace(B: int, K: int, N: int) -> int:
    return lib().scap_fc_host_workspace(B, K, N)


def scap_sparse_fc_host(x_host, W, m, tau, b_fused, y_host, ws, stream=None) -> None:
    """x_host / y_host are CPU tensors (pinned recommended); everything else lives on the device."""
    B, K = x_host.shape
    N = W.shape[1]
    p, n = _ws(ws)
    _invoke("scap_sparse_fc_host", x_host, W, m, tau, b_fused, y_host, B, K, N, dtype_of(W), p, n, _stream(stream))


def scap_glu_workspace(B: int, D: int, F: int) -> int:
    return lib().scap_glu_workspace(B, D, F)


def scap_glu_ffn(h, Wgu, Wd, m1, tau1, bgu_fused, m2, tau2, bd_fused, y, ws, z_out=None, idx1_out=None, nnz1_out=None,
                 idx2_out=None, nnz2_out=None, stream=None) -> None:
    B, D = h.shape
    F = Wd.shape[0]
    p, n = _ws(ws)
    _invoke("scap_glu_ffn", h, Wgu, Wd, m1, tau1, bgu_fused, m2, tau2, bd_fused, y, B, D, F, dtype_of(Wgu), z_out, idx1_out, nnz1_out,
            idx2_out, nnz2_out, p, n, _stream(stream))


def scap_gelu_ffn_workspace(B: int, D: int, F: int) -> int:
    return lib().scap_gelu_ffn_workspace(B, D, F)


def scap_gelu_ffn(h, Wu, Wd, m1, tau1, bu_fused, m2, tau2, bd_fused, y, ws, z_out=None, idx1_out=None, nnz1_out=None,
                  idx2_out=None, nnz2_out=None, stream=None) -> None:
    B, D = h.shape
    F = Wd.shape[0]
    p, n = _ws(ws)
    _invoke("scap_gelu_ffn", h, Wu, Wd, m1, tau1, bu_fused, m2, tau2, bd_fused, y, B, D, F, dtype_of(Wu), z_out, idx1_out, nnz1_out,
            idx2_out, nnz2_out, p, n, _stream(stream))


def scap_glu_static_capacity() -> int:
    return lib().scap_glu_static_capacity()


def scap_glu_ffn_static(h, Wgu, Wd, m1, tau1, bgu_fused, m2, tau2, bd_fused, y, z_out=None, stream=None) -> None:
    """scap_glu_ffn for callers that may not allocate: the scratch is a fixed array inside the library (see scap.h)."""
    B, D = h.shape
    F = Wd.shape[0]
    _invoke("scap_glu_ffn_static", h, Wgu, Wd, m1, tau1, bgu_fused, m2, tau2, bd_fused, y, B, D, F, dtype_of(Wgu), z_out, _stream(stream))


def scap_moe_workspace(B: int, D: int, F: int, E: int, top_k: int) -> int:
    return lib().scap_moe_workspace(B, D, F, E, top_k)


def scap_moe_ffn(h, logits, experts, top_k: int, y, ws, expert_out=None, weight_out=None, stream=None) -> None:
    """``experts``: list of dicts of tensors with the fields of ``scap_expert`` (None where nullable)."""
    B, D = h.shape
    E = len(experts)
    F = experts[0]["Wd"].shape[0]
    arr = (ScapExpert * E)()
    for e, p_ in enumerate(experts):
        for name, _ in ScapExpert._fields_:
            setattr(arr[e], name, _ptr(p_.get(name)))
    p, n = _ws(ws)
    _check(lib().scap_moe_ffn(_ptr(h), _ptr(logits), arr, E, top_k, _ptr(y), B, D, F, dtype_of(h), _ptr(expert_out),
                              _ptr(weight_out), p, n, _stream(stream)), "scap_moe_ffn")


_getDevice, _getCurrentRawStream = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_on(device: int, stream, *tensors) -> int:
    """The stream of a call whose tensors have to be on one device, the current one (device: the number of that, -1 for none): memory of another one, or of
    the host, is out of a kernel's reach."""
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on one device")
    if device < 0:
        return _stream(stream)
    if device != _getDevice():
        raise ValueError("the tensors are on device %d, which is not the current one" % device)
    return _getCurrentRawStream(device) if stream is None else _stream(stream)


def _rows(t, rows: int, cols: int, name: str) -> int:
    """Row stride of a matrix [rows, cols] whose rows are contiguous, in elements."""
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError("%s must have contiguous rows" % name)
    return ld if rows > 1 else max(ld, cols)


def scap_fc_act_workspace(M: int, K: int, N: int, ldx: int | None = None) -> int:
    return lib().scap_fc_act_workspace(M, K, N, K if ldx is None else ldx)


def scap_fc_act(x, W, b, y, ws, act: int = SCAP_ACT_NONE, res=None, stream=None) -> None:
    """y = act(x W + b) + res on any number of rows; rows of x, res and y may lie apart (views of wider matrices)."""
    M, K = x.shape
    K_, N = shape = W.shape
    dt = dtype_of(x)
    ydt = SCAP_F32 if y.dtype is torch.float32 else dtype_of(y)
    if x.dtype is not W.dtype or K_ != K or not W.is_contiguous() or y.shape != (M, N):
        raise ValueError("x [M, K] and W [K, N] must have one dtype, W contiguous rows, y the shape [M, N]: %s" % (shape,))
    if b is not None and (b.dtype is not torch.float32 or b.numel() != N or not b.is_contiguous()):
        raise ValueError("b must be float32 [N]")
    ldr = 0
    if res is not None:
        if res.dtype is not y.dtype or res.shape != (M, N):
            raise ValueError("res must have the shape and dtype of y")
        ldr = _rows(res, M, N, "res")
    stream = _stream_on(x.get_device(), stream, W, b, y, ws, res)
    p, n = _ws(ws)
    _invoke("scap_fc_act", x, _rows(x, M, K, "x"), W, b, int(act), res, ldr, y, _rows(y, M, N, "y"), M, K, N, dt, ydt, p, n, stream)


class ScapKv4(C.Structure):
    """The 4-bit cache of one layer (``scap_kv4``), made of the tensors that hold it.  ``pages`` [n_pages, bytes] uint8 may be a
    view of wider pages (several layers side by side), but the calls that copy pages want the pool itself; ``table`` [n_seqs, pages of a sequence], ``lens`` [n_seqs] and ``refs`` [n_pages] are int32."""
    _fields_ = [("pages", C.c_void_p), ("page_stride", C.c_size_t), ("n_pages", C.c_int), ("page_tokens", C.c_int), ("heads", C.c_int),
                ("head_dim", C.c_int), ("group", C.c_int), ("table_stride", C.c_int), ("n_seqs", C.c_int), ("table", C.c_void_p),
                ("lens", C.c_void_p), ("refs", C.c_void_p)]

    def __init__(self, pages, page_tokens: int, heads: int, head_dim: int, group: int, table, lens, refs=None):
        n_pages, width = pages.shape
        n_seqs, row = table.shape
        stride, one = pages.stride()
        if pages.dtype is not torch.uint8 or one != 1:
            raise ValueError("pages must be uint8 [n_pages, bytes] with contiguous rows")
        if table.dtype is not torch.int32 or not table.is_contiguous():
            raise ValueError("table must be contiguous int32 [n_seqs, pages of a sequence]")
        if lens.dtype is not torch.int32 or lens.shape != (n_seqs,) or not lens.is_contiguous():
            raise ValueError("lens must be contiguous int32 [%d]" % n_seqs)
        if refs is not None and (refs.dtype is not torch.int32 or refs.shape != (n_pages,) or not refs.is_contiguous()):
            raise ValueError("refs must be contiguous int32 [%d]" % n_pages)
        device = pages.get_device()
        if table.get_device() != device or lens.get_device() != device or (refs is not None and refs.get_device() != device):
            raise ValueError("pages, table, lens and refs must be on one device")
        if heads and width < scap_kv4_page_bytes(page_tokens, heads, head_dim, group):
            raise ValueError("a page needs %d bytes, has %d" % (scap_kv4_page_bytes(page_tokens, heads, head_dim, group), width))
        super().__init__(pages.data_ptr(), stride if n_pages > 1 else max(stride, width), n_pages, page_tokens, heads, head_dim, group, row, n_seqs, table.data_ptr(),
                         lens.data_ptr(), None if refs is None else refs.data_ptr())
        self.tensors = (pages, table, lens, refs)  # kept alive with the description
        # whole pages (bytes): rows of the matrix that `pages` is, or is a slice of
        self.whole = width == self.page_stride or (pages.storage_offset() % self.page_stride == 0 and
                                         pages.storage_offset() + n_pages * self.page_stride <= pages.untyped_storage().nbytes())
        self.address = C.addressof(self)
        self.device = device
        self.shape = (n_seqs, heads, head_dim)


def scap_kv4_page_bytes(page_tokens: int, heads: int, head_dim: int, group: int) -> int:
    return lib().scap_kv4_page_bytes(int(page_tokens), int(heads), int(head_dim), int(group))


def _tokens(t, rows: int, heads: int, D: int, name: str) -> int:
    """Elements between the tokens of [rows, heads, D], which may be a slice of a wider row."""
    ld, of_head, one = t.stride()
    if one != 1 or (heads > 1 and of_head != D):
        raise ValueError("%s must be [tokens, %d, %d] with contiguous heads" % (name, heads, D))
    return ld if rows > 1 else max(ld, heads * D)


def _kv4_rows(name: str, cache, k, v, row_start, stream) -> None:
    n_seqs, heads, D = cache.shape
    rows = k.shape[0]
    if k.shape != (rows, heads, D) or v.shape != (rows, heads, D) or k.dtype is not v.dtype:
        raise ValueError("k and v must be [rows, %d, %d] of one dtype" % (heads, D))
    if row_start is not None and (row_start.dtype is not torch.int32 or row_start.numel() != n_seqs + 1 or not row_start.is_contiguous()):
        raise ValueError("row_start must be int32 [n_seqs + 1]")
    stream = _stream_on(cache.device, stream, k, v, row_start)
    _invoke(name, cache.address, k, _tokens(k, rows, heads, D, "k"), v, _tokens(v, rows, heads, D, "v"), row_start, rows, dtype_of(k), stream)


def scap_kv4_append(cache, k, v, row_start=None, stream=None) -> None:
    """Stores new tokens k, v [rows, heads, head_dim] as the last tokens of their sequences (``cache.lens`` includes them)."""
    _kv4_rows("scap_kv4_append", cache, k, v, row_start, stream)


def scap_kv4_read(cache, k_out, v_out, row_start=None, stream=None) -> None:
    """The values that the cache holds for the last tokens of its sequences, addressed as in scap_kv4_append."""
    _kv4_rows("scap_kv4_read", cache, k_out, v_out, row_start, stream)


def scap_kv4_attend_workspace(n_seqs: int, nq: int, q_heads: int, heads: int, head_dim: int) -> int:
    return lib().scap_kv4_attend_workspace(int(n_seqs), int(nq), int(q_heads), int(heads), int(head_dim))


def _queries(t, n_seqs: int, nq: int, heads: int, D: int, name: str) -> int:
    """Elements between the tokens of [n_seqs, nq, heads, D], which may be a slice of a wider row."""
    of_seq, ld, of_head, one = t.stride()
    if one != 1 or (heads > 1 and of_head != D) or (n_seqs > 1 and nq > 1 and of_seq != nq * ld):
        raise ValueError("%s must have contiguous heads, and evenly spaced tokens" % name)
    return ld if nq > 1 else (of_seq if n_seqs > 1 else heads * D)


def scap_kv4_attend(cache, q, out, scale: float, ws, window: int = 0, lse=None, stream=None) -> None:
    """out[b, i, h]: attention of the last nq tokens of every sequence, q [n_seqs, nq, q_heads, head_dim], over its tokens in the cache."""
    n_seqs, _, D = cache.shape
    shape = q.shape
    B, nq, heads, D_ = shape
    if B != n_seqs or D_ != D or out.shape != shape or out.dtype is not q.dtype:
        raise ValueError("q and out must be [%d, nq, q_heads, %d] of one dtype" % (n_seqs, D))
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (B, nq, heads) or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [n_seqs, nq, q_heads]")
    stream = _stream_on(cache.device, stream, q, out, lse, ws)
    p, n = _ws(ws)
    _invoke_real("scap_kv4_attend", float(scale), 8, cache.address, q, _queries(q, B, nq, heads, D, "q"), out, _queries(out, B, nq, heads, D, "out"), lse, nq, heads, int(window),
                 dtype_of(q), p, n, stream)


def scap_kv4_pages_workspace(n_pages: int, n: int) -> int:
    return lib().scap_kv4_pages_workspace(int(n_pages), int(n))


def _numbers(name: str, device: int, *tensors) -> int:
    """Length that the int32 tensors share."""
    n = tensors[0].numel()
    for t in tensors:
        if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
            raise ValueError("%s must be contiguous int32 tensors of one length on the device of the cache" % name)
    return n


def _count(t, name: str, device: int):
    """Where a count goes: an int32 tensor of one element or more, an address or None."""
    if t is not None and type(t) is not int and (t.dtype is not torch.int32 or t.get_device() != device or t.numel() < 1):
        raise ValueError("%s must be int32 [1] on the device of the cache" % name)
    return t


_WHOLE = "pages move whole, all page_stride bytes: the cache must be described by the pool, not by a layer inside its pages"


def scap_kv4_copy(cache, src, dst, stream=None) -> None:
    """Copies page src[i] to page dst[i]."""
    if not cache.whole:
        raise ValueError(_WHOLE)
    device = cache.device
    _invoke("scap_kv4_copy", cache.address, src, dst, _numbers("src and dst", device, src, dst), _stream_on(device, stream))


def scap_kv4_fork(cache, src, dst, fail, ws, stream=None) -> None:
    """Row dst[i] becomes a copy of row src[i]: full pages shared, the last one copied.  fail [1] int32 or None: requests not carried out."""
    if not cache.whole:
        raise ValueError(_WHOLE)
    device = cache.device
    p, n = _ws(ws)
    _invoke("scap_kv4_fork", cache.address, src, dst, _numbers("src and dst", device, src, dst), _count(fail, "fail", device), p, n, _stream_on(device, stream, ws))


def scap_kv4_free(cache, rows, stream=None) -> None:
    """Lets go the pages of the rows; the rows are empty after it."""
    device = cache.device
    _invoke("scap_kv4_free", cache.address, rows, _numbers("rows", device, rows), _stream_on(device, stream))


def scap_kv4_reserve(cache, add, fail, ws, stream=None) -> None:
    """lens[b] += add[b], with free pages for the new tokens.  fail [1] int32 or None: sequences that did not get them."""
    device = cache.device
    if _numbers("add", device, add) != cache.shape[0]:
        raise ValueError("add must be int32 [n_seqs]")
    p, n = _ws(ws)
    _invoke("scap_kv4_reserve", cache.address, add, _count(fail, "fail", device), p, n, _stream_on(device, stream, ws))


def scap_kv4_compact(cache, used, ws, stream=None) -> None:
    """Moves the used pages to the front of the pool; used [1] int32 or None: how many there are."""
    if not cache.whole:
        raise ValueError(_WHOLE)
    device = cache.device
    p, n = _ws(ws)
    _invoke("scap_kv4_compact", cache.address, _count(used, "used", device), p, n, _stream_on(device, stream, ws))
