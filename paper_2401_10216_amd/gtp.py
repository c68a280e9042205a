"""Thin ctypes binding of libgtp.so (the C ABI in include/gtp.h).

Only argument marshalling happens here: every step of the Gaunt tensor
product runs in the library's HIP kernels.  Tensors are torch CUDA (HIP)
tensors; the current torch stream is passed to the library.  If the library
is not built the import of any entry point raises -- there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
import threading

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libgtp.so")

GTP_OK, GTP_ERR_INVALID_ARG, GTP_ERR_UNSUPPORTED, GTP_ERR_NO_DEVICE, GTP_ERR_HIP, GTP_ERR_ALLOC = range(6)
GTP_F32, GTP_BF16 = 0, 1
GTP_CONV_AUTO, GTP_CONV_DIRECT, GTP_CONV_FFT, GTP_CONV_DFT = 0, 1, 2, 3
GTP_PLAN_HOST_ONLY = 16
GTP_FORCE_GENERIC = 32  # internal: use the workgroup-per-product kernel
GTP_SELF_STEPWISE, GTP_SELF_FUSED = 0, 1

_lib = None
_lock = threading.Lock()


class GTPError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


_STATUS = {0: "GTP_OK", 1: "GTP_ERR_INVALID_ARG", 2: "GTP_ERR_UNSUPPORTED", 3: "GTP_ERR_NO_DEVICE",
           4: "GTP_ERR_HIP", 5: "GTP_ERR_ALLOC"}

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I = ctypes.c_int
_U = ctypes.c_uint
_DP = ctypes.POINTER(ctypes.c_double)



class _Rows(ctypes.Structure):
    """gtp_rows."""
    _fields_ = [("data", _P), ("row", _I64), ("head", _I64)]


class _Attn(ctypes.Structure):
    """gtp_attn."""
    _fields_ = [("dtype", _I), ("H", _I), ("Hk", _I), ("d", _I), ("B", _I64), ("Tq", _I64), ("Tk", _I64),
                ("max_q", _I64), ("max_k", _I64), ("q_off", _P), ("k_off", _P), ("key_mask", _P),
                ("scale", ctypes.c_float), ("p", ctypes.c_double), ("rng", _P)]


# The same layouts to pack a call's structs with (a Structure's fields one by one take several times as long).
_ATTN = struct.Struct("<4i5q3Qf4xdQ")
_ROWS = "Qqq"
assert _ATTN.size == ctypes.sizeof(_Attn) and struct.calcsize("<" + _ROWS) == ctypes.sizeof(_Rows)

_SIGS = {
    "gtp_plan_create": (_I, [ctypes.POINTER(_P), _I, _I, _I, _U]),
    "gtp_plan_destroy": (_I, [_P]),
    "gtp_full": (_I, [_P, _P, _P, _I, _I64, _I64, _P, _P]),
    "gtp_full_backward": (_I, [_P, _P, _P, _I, _P, _I64, _I64, _P, _P, _P]),
    "gtp_full_weighted": (_I, [_P, _P, _P, _I, _P, _P, _P, _I, _I64, _I64, _P, _P]),
    "gtp_full_weighted_backward": (_I, [_P, _P, _P, _I, _P, _P, _P, _I, _P, _I64, _I64, _P, _P, _P, _P, _P, _P]),
    "gtp_conv_escn": (_I, [_P, _P, _I, _P, _P, _I64, _I64, _P, _P]),
    "gtp_conv_escn_noalloc": (_I, [_P, _P, _I, _P, _P, _I64, _I64, _P, _P]),
    "gtp_channel_mix": (_I, [_P, _P, _P, _I, _P, _I64, _I64, _I64, _I64, _P, _P]),
    "gtp_sh2fourier": (_I, [_P, _I, _P, _I, _I64, _P, _P]),
    "gtp_fourier_conv": (_I, [_P, _P, _P, _I64, _P, _P]),
    "gtp_fourier2sh": (_I, [_P, _P, _I64, _P, _P]),
    "gtp_selfproduct": (_I, [_I, _I, _I, _U, _P, _I, _I64, _I64, _P, _P]),
    "gtp_sh_filter": (_I, [_I, _P, _P, _I64, _I64, _P, _P]),
    "gtp_layer_norm": (_I, [_I, _P, _I, _P, _P, ctypes.c_float, _I64, _I64, _P, _P, _P, _P]),
    "gtp_layer_norm_backward_work": (_I64, [_I, _I, _I64, _I64]),
    "gtp_layer_norm_backward": (_I, [_I, _P, _I, _P, _P, _P, _P, _I64, _I64, _P, _P, _P, _P, _I64, _P]),
    "gtp_dropout": (_I, [_P, _P, _I, ctypes.c_double, _P, _I64, _I64, _P, _P]),
    "gtp_attention_work": (_I64, [_P, _I]),
    "gtp_attention": (_I, [_P, _P, _P, _P, _P, _P, _P, _I64, _P]),
    "gtp_attention_backward": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _P]),
    "gtp_stream_probe": (_I, [_I, _P, _P, _I64, _P]),
    "gtp_compute_probe": (_I, [_I, _I64, _P, _DP, _P]),
    "gtp_grid_floats": (_I64, [_P, _I]),
    "gtp_plan_info": (_I, [_P, ctypes.POINTER(_I64)]),
    "gtp_plan_table": (_I, [_P, _I, _DP, ctypes.POINTER(_I64)]),
    "gtp_debug_host_pipeline": (_I, [_P, _DP, _DP, _I64, _DP]),
    "gtp_status_str": (ctypes.c_char_p, [_I]),
    "gtp_last_error": (ctypes.c_char_p, []),
}


def _load(path: str):
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2401_10216_amd.build`")
    L = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    return L


def lib():
    """Load libgtp.so once (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is None:
            _lib = _load(LIB_PATH)
    return _lib


class use_library:
    """Context in which the entry points (and the plans created there) use
    another build of the library, e.g. the poisoned-LDS debug build
    (libgtp_poison.so).  A plan keeps the library it was created with."""

    def __init__(self, path: str):
        self.path = path

    def __enter__(self):
        global _lib
        with _lock:
            self.saved = _lib
            _lib = _load(self.path)
        return _lib

    def __exit__(self, *exc):
        global _lib
        with _lock:
            _lib = self.saved
        return False


def _check(status: int, L=None):
    if status != GTP_OK:
        raise GTPError(status, (L or lib()).gtp_last_error().decode())


def _stream(stream=None):
    import torch
    if stream is None and torch.cuda.is_initialized():
        # the current stream's handle without a Stream object around it (several us a call), where torch has that
        # function: its name is not one that torch promises
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return ctypes.c_void_p(raw(torch.cuda.current_device()))
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return GTP_F32
    if t.dtype == torch.bfloat16:
        return GTP_BF16
    raise TypeError(f"unsupported input dtype {t.dtype} (float32 or bfloat16)")


def _dev(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _want(t, name, shape, dtypes, device=None):
    """Validate a caller-supplied tensor before anything reaches the library:
    exact shape, one of the allowed dtypes, contiguous, on the device of the
    other operands.  Raises TypeError (dtype) or ValueError (everything else)
    and returns the tensor's device pointer."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}; expected " + " or ".join(str(d) for d in dtypes))
    if t.shape != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}; expected {tuple(int(v) for v in shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}; the other operands are on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _on_gpu(t, name):
    """Last check before a call: the operands (all on t's device) are device tensors."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _f32():
    import torch
    return (torch.float32,)


def _inputs():
    import torch
    return (torch.float32, torch.bfloat16)


def nsh(L: int) -> int:
    return (L + 1) * (L + 1)


class Plan:
    """gtp_plan_create / gtp_plan_destroy."""

    def __init__(self, L1: int, L2: int, Lout: int, flags: int = 0):
        self.L1, self.L2, self.Lout, self.flags = L1, L2, Lout, flags
        h = _P()
        self.lib = lib()
        _check(self.lib.gtp_plan_create(ctypes.byref(h), L1, L2, Lout, flags), self.lib)
        self.handle = h

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.gtp_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def info(self) -> dict:
        out = (_I64 * 8)()
        _check(self.lib.gtp_plan_info(self.handle, out), self.lib)
        keys = ["L1", "L2", "Lout", "U", "Le", "NT", "NP", "conv"]
        return dict(zip(keys, [int(v) for v in out]))

    def table(self, which: int):
        import numpy as np
        cnt = _I64(0)
        _check(self.lib.gtp_plan_table(self.handle, which, None, ctypes.byref(cnt)), self.lib)
        buf = np.zeros(cnt.value, dtype=np.float64)
        _check(self.lib.gtp_plan_table(self.handle, which, buf.ctypes.data_as(_DP), ctypes.byref(cnt)), self.lib)
        return buf

    def grid_floats(self, which: int) -> int:
        return int(self.lib.gtp_grid_floats(self.handle, which))


def gtp_full(plan: Plan, x1, x2, y=None, stream=None):
    """y[B,C,(Lout+1)^2] = Gaunt tensor product of x1[B,C,(L1+1)^2] and x2[B,C,(L2+1)^2]."""
    import torch
    if x1.dtype != x2.dtype:
        raise TypeError("x1 and x2 must have the same dtype")
    if x1.dim() != 3 or x2.dim() != 3 or x1.shape[:2] != x2.shape[:2]:
        raise ValueError("x1, x2 must be [B, C, K] with equal B, C")
    if x1.shape[2] != nsh(plan.L1) or x2.shape[2] != nsh(plan.L2):
        raise ValueError("coefficient dimension does not match the plan")
    B, C = int(x1.shape[0]), int(x1.shape[1])
    code = _dtype_code(x1)
    p1 = _want(x1, "x1", x1.shape, _inputs())
    p2 = _want(x2, "x2", x2.shape, _inputs(), x1.device)
    if y is None:
        y = torch.empty((B, C, nsh(plan.Lout)), dtype=torch.float32, device=x1.device)
    py = _want(y, "y", (B, C, nsh(plan.Lout)), _f32(), x1.device)
    _on_gpu(x1, "x1")
    _check(plan.lib.gtp_full(plan.handle, p1, p2, code, B, C, py, _stream(stream)), plan.lib)
    return y


def gtp_channel_mix(plan: Plan, x1, x2, W, y=None, stream=None):
    """y[B,Co,(Lout+1)^2] = sum_{c1,c2} W[co,c1,c2] GTP(x1[:,c1], x2[:,c2]); W float32 [Co, C1, C2]."""
    import torch
    if x1.dtype != x2.dtype:
        raise TypeError("x1 and x2 must have the same dtype")
    if x1.dim() != 3 or x2.dim() != 3 or x1.shape[0] != x2.shape[0]:
        raise ValueError("x1 [B, C1, K1] and x2 [B, C2, K2] with equal B")
    if x1.shape[2] != nsh(plan.L1) or x2.shape[2] != nsh(plan.L2):
        raise ValueError("coefficient dimension does not match the plan")
    B, C1, C2 = int(x1.shape[0]), int(x1.shape[1]), int(x2.shape[1])
    if W.dim() != 3 or tuple(W.shape[1:]) != (C1, C2) or W.dtype != torch.float32:
        raise ValueError("W must be float32 [Co, C1, C2]")
    Co = int(W.shape[0])
    code = _dtype_code(x1)
    p1 = _want(x1, "x1", x1.shape, _inputs())
    p2 = _want(x2, "x2", x2.shape, _inputs(), x1.device)
    pw = _want(W, "W", (Co, C1, C2), _f32(), x1.device)
    if y is None:
        y = torch.empty((B, Co, nsh(plan.Lout)), dtype=torch.float32, device=x1.device)
    py = _want(y, "y", (B, Co, nsh(plan.Lout)), _f32(), x1.device)
    _on_gpu(x1, "x1")
    _check(plan.lib.gtp_channel_mix(plan.handle, p1, p2, code, pw, B, C1, C2, Co, py, _stream(stream)), plan.lib)
    return y


def gtp_conv_escn(plan: Plan, x, r, h, y=None, stream=None, noalloc: bool = False):
    """y[B,C,(Lout+1)^2] = GTP(x, h[b,c,l] Y_l(r_b / |r_b|)) in the edge's rotated frame; r [B, 3], h [B, C, L2+1] fp32.
    noalloc=True calls gtp_conv_escn_noalloc (static device scratch, no allocation by the library; y must then be
    given for no allocation to happen at all)."""
    import torch
    if x.dim() != 3 or x.shape[2] != nsh(plan.L1):
        raise ValueError("x must be [B, C, (L1+1)^2]")
    B, C = int(x.shape[0]), int(x.shape[1])
    if tuple(r.shape) != (B, 3) or r.dtype != torch.float32:
        raise ValueError("r must be float32 [B, 3]")
    if tuple(h.shape) != (B, C, plan.L2 + 1) or h.dtype != torch.float32:
        raise ValueError("h must be float32 [B, C, L2+1]")
    code = _dtype_code(x)
    px = _want(x, "x", x.shape, _inputs())
    pr = _want(r, "r", (B, 3), _f32(), x.device)
    ph = _want(h, "h", (B, C, plan.L2 + 1), _f32(), x.device)
    if y is None:
        y = torch.empty((B, C, nsh(plan.Lout)), dtype=torch.float32, device=x.device)
    py = _want(y, "y", (B, C, nsh(plan.Lout)), _f32(), x.device)
    _on_gpu(x, "x")
    fn = plan.lib.gtp_conv_escn_noalloc if noalloc else plan.lib.gtp_conv_escn
    _check(fn(plan.handle, px, code, pr, ph, B, C, py, _stream(stream)), plan.lib)
    return y


def gtp_full_weighted(plan: Plan, x1, x2, w1=None, w2=None, wout=None, per_channel: bool = False, y=None,
                      stream=None):
    """y = wout * GTP(w1 * x1, w2 * x2) with per-degree weights w1[R, L1+1], w2[R, L2+1], wout[R, Lout+1]
    (fp32 device tensors or None = ones; R = C if per_channel else 1)."""
    import torch
    if x1.dtype != x2.dtype:
        raise TypeError("x1 and x2 must have the same dtype")
    if x1.dim() != 3 or x2.dim() != 3 or x1.shape[:2] != x2.shape[:2]:
        raise ValueError("x1, x2 must be [B, C, K] with equal B, C")
    if x1.shape[2] != nsh(plan.L1) or x2.shape[2] != nsh(plan.L2):
        raise ValueError("coefficient dimension does not match the plan")
    B, C = int(x1.shape[0]), int(x1.shape[1])
    R = C if per_channel else 1
    ptrs = []
    for w, L, name in ((w1, plan.L1, "w1"), (w2, plan.L2, "w2"), (wout, plan.Lout, "wout")):
        if w is None:
            ptrs.append(ctypes.c_void_p(None))
            continue
        ptrs.append(_want(w, name, (R, L + 1), _f32(), x1.device))
    code = _dtype_code(x1)
    p1 = _want(x1, "x1", x1.shape, _inputs())
    p2 = _want(x2, "x2", x2.shape, _inputs(), x1.device)
    if y is None:
        y = torch.empty((B, C, nsh(plan.Lout)), dtype=torch.float32, device=x1.device)
    py = _want(y, "y", (B, C, nsh(plan.Lout)), _f32(), x1.device)
    _on_gpu(x1, "x1")
    _check(plan.lib.gtp_full_weighted(plan.handle, p1, p2, code, *ptrs, 1 if per_channel else 0, B, C, py,
                                      _stream(stream)), plan.lib)
    return y


def gtp_full_weighted_backward(plan: Plan, x1, x2, dy, w1=None, w2=None, wout=None, per_channel: bool = False,
                               need=("dx1", "dx2", "dw1", "dw2", "dwout"), stream=None):
    """Gradients of <dy, gtp_full_weighted(x1, x2, w1, w2, wout)>: a dict with the requested keys among dx1, dx2
    ([B, C, K] fp32) and dw1, dw2, dwout ([R, L+1] fp32, R = C if per_channel else 1)."""
    import torch
    if x1.dtype != x2.dtype:
        raise TypeError("x1 and x2 must have the same dtype")
    if x1.dim() != 3 or x2.dim() != 3 or x1.shape[:2] != x2.shape[:2]:
        raise ValueError("x1, x2 must be [B, C, K] with equal B, C")
    if x1.shape[2] != nsh(plan.L1) or x2.shape[2] != nsh(plan.L2):
        raise ValueError("coefficient dimension does not match the plan")
    unknown = set(need) - {"dx1", "dx2", "dw1", "dw2", "dwout"}
    if unknown:
        raise ValueError(f"unknown gradients {sorted(unknown)}")
    B, C = int(x1.shape[0]), int(x1.shape[1])
    R = C if per_channel else 1
    code = _dtype_code(x1)
    px1 = _want(x1, "x1", x1.shape, _inputs())
    px2 = _want(x2, "x2", x2.shape, _inputs(), x1.device)
    pdy = _want(dy, "dy", (B, C, nsh(plan.Lout)), _f32(), x1.device)
    ws = []
    for w, L, name in ((w1, plan.L1, "w1"), (w2, plan.L2, "w2"), (wout, plan.Lout, "wout")):
        ws.append(ctypes.c_void_p(None) if w is None else _want(w, name, (R, L + 1), _f32(), x1.device))
    shapes = {"dx1": (B, C, nsh(plan.L1)), "dx2": (B, C, nsh(plan.L2)), "dw1": (R, plan.L1 + 1),
              "dw2": (R, plan.L2 + 1), "dwout": (R, plan.Lout + 1)}
    out = {k: torch.empty(shapes[k], dtype=torch.float32, device=x1.device) for k in need}
    ptr = {k: (ctypes.c_void_p(out[k].data_ptr()) if k in out else ctypes.c_void_p(None)) for k in shapes}
    _on_gpu(x1, "x1")
    _check(plan.lib.gtp_full_weighted_backward(plan.handle, px1, px2, code, *ws, 1 if per_channel else 0, pdy, B, C,
                                               ptr["dx1"], ptr["dx2"], ptr["dw1"], ptr["dw2"], ptr["dwout"],
                                               _stream(stream)), plan.lib)
    return out


def gtp_full_backward(plan: Plan, x1, x2, dy, need_dx1: bool = True, need_dx2: bool = True, dx1=None, dx2=None,
                      stream=None):
    """(dx1, dx2): gradients of <dy, gtp_full(x1, x2)> in x1 and x2 (fp32; None when not requested)."""
    import torch
    if x1.dtype != x2.dtype:
        raise TypeError("x1 and x2 must have the same dtype")
    if x1.dim() != 3 or x2.dim() != 3 or dy.dim() != 3 or x1.shape[:2] != x2.shape[:2] or dy.shape[:2] != x1.shape[:2]:
        raise ValueError("x1, x2, dy must be [B, C, K] with equal B, C")
    if x1.shape[2] != nsh(plan.L1) or x2.shape[2] != nsh(plan.L2) or dy.shape[2] != nsh(plan.Lout):
        raise ValueError("coefficient dimension does not match the plan")
    if dy.dtype != torch.float32:
        raise TypeError("dy must be float32")
    B, C = int(x1.shape[0]), int(x1.shape[1])
    code = _dtype_code(x1)
    px1 = _want(x1, "x1", x1.shape, _inputs())
    px2 = _want(x2, "x2", x2.shape, _inputs(), x1.device)
    pdy = _want(dy, "dy", (B, C, nsh(plan.Lout)), _f32(), x1.device)
    if need_dx1 and dx1 is None:
        dx1 = torch.empty((B, C, nsh(plan.L1)), dtype=torch.float32, device=x1.device)
    if need_dx2 and dx2 is None:
        dx2 = torch.empty((B, C, nsh(plan.L2)), dtype=torch.float32, device=x1.device)
    p1 = _want(dx1, "dx1", (B, C, nsh(plan.L1)), _f32(), x1.device) if need_dx1 else ctypes.c_void_p(None)
    p2 = _want(dx2, "dx2", (B, C, nsh(plan.L2)), _f32(), x1.device) if need_dx2 else ctypes.c_void_p(None)
    _on_gpu(x1, "x1")
    _check(plan.lib.gtp_full_backward(plan.handle, px1, px2, code, pdy, B, C, p1, p2, _stream(stream)), plan.lib)
    return (dx1 if need_dx1 else None), (dx2 if need_dx2 else None)


def gtp_sh2fourier(plan: Plan, which: int, x, grid=None, stream=None):
    """Complex grids [n, 2L+1, 2L+1] (as torch.complex64) of x[n, (L+1)^2]."""
    import torch
    if which not in (1, 2):
        raise ValueError("which must be 1 or 2")
    L = plan.L1 if which == 1 else plan.L2
    if x.dim() != 2:
        raise ValueError("x must be [n, (L+1)^2]")
    n = int(x.shape[0])
    code = _dtype_code(x)
    px = _want(x, "x", (n, nsh(L)), _inputs())
    if grid is None:
        grid = torch.empty((n, 2 * L + 1, 2 * L + 1), dtype=torch.complex64, device=x.device)
    pg = _want(grid, "grid", (n, 2 * L + 1, 2 * L + 1), (torch.complex64,), x.device)
    _on_gpu(x, "x")
    _check(plan.lib.gtp_sh2fourier(plan.handle, which, px, code, n, pg, _stream(stream)), plan.lib)
    return grid


def gtp_fourier_conv(plan: Plan, g1, g2, g3=None, stream=None):
    import torch
    if g1.dim() != 3:
        raise ValueError("g1 must be [n, 2 L1 + 1, 2 L1 + 1]")
    n = int(g1.shape[0])
    D1, D2, D3 = 2 * plan.L1 + 1, 2 * plan.L2 + 1, 2 * (plan.L1 + plan.L2) + 1
    c64 = (torch.complex64,)
    p1 = _want(g1, "g1", (n, D1, D1), c64)
    p2 = _want(g2, "g2", (n, D2, D2), c64, g1.device)
    if g3 is None:
        g3 = torch.empty((n, D3, D3), dtype=torch.complex64, device=g1.device)
    p3 = _want(g3, "g3", (n, D3, D3), c64, g1.device)
    _on_gpu(g1, "g1")
    _check(plan.lib.gtp_fourier_conv(plan.handle, p1, p2, n, p3, _stream(stream)), plan.lib)
    return g3


def gtp_fourier2sh(plan: Plan, g3, y=None, stream=None):
    import torch
    if g3.dim() != 3:
        raise ValueError("g3 must be [n, 2U + 1, 2U + 1]")
    n = int(g3.shape[0])
    D3 = 2 * (plan.L1 + plan.L2) + 1
    p3 = _want(g3, "g3", (n, D3, D3), (torch.complex64,))
    if y is None:
        y = torch.empty((n, nsh(plan.Lout)), dtype=torch.float32, device=g3.device)
    py = _want(y, "y", (n, nsh(plan.Lout)), _f32(), g3.device)
    _on_gpu(g3, "g3")
    _check(plan.lib.gtp_fourier2sh(plan.handle, p3, n, py, _stream(stream)), plan.lib)
    return y


def gtp_selfproduct(x, L: int, nu: int, Lout: int, mode: int = GTP_SELF_STEPWISE, y=None, stream=None):
    import torch
    if x.dim() != 3 or x.shape[2] != nsh(L):
        raise ValueError("x must be [B, C, (L+1)^2]")
    B, C = int(x.shape[0]), int(x.shape[1])
    code = _dtype_code(x)
    px = _want(x, "x", x.shape, _inputs())
    if y is None:
        y = torch.empty((B, C, nsh(Lout)), dtype=torch.float32, device=x.device)
    py = _want(y, "y", (B, C, nsh(Lout)), _f32(), x.device)
    _on_gpu(x, "x")
    _check(lib().gtp_selfproduct(L, nu, Lout, mode, px, code, B, C, py, _stream(stream)))
    return y


def gtp_sh_filter(L: int, r, h=None, out=None, stream=None):
    """out[B,C,(L+1)^2] = h[B,C,L+1] * Y(r_b); h=None gives Y(r) with C = 1."""
    import torch
    if r.dim() != 2:
        raise ValueError("r must be [B, 3]")
    B = int(r.shape[0])
    pr = _want(r, "r", (B, 3), _f32())
    if h is not None and h.dim() != 3:
        raise ValueError("h must be [B, C, L+1]")
    C = 1 if h is None else int(h.shape[1])
    hp = ctypes.c_void_p(None) if h is None else _want(h, "h", (B, C, L + 1), _f32(), r.device)
    if out is None:
        out = torch.empty((B, C, nsh(L)), dtype=torch.float32, device=r.device)
    po = _want(out, "out", (B, C, nsh(L)), _f32(), r.device)
    _on_gpu(r, "r")
    _check(lib().gtp_sh_filter(L, pr, hp, B, C, po, _stream(stream)))
    return out


_HERE = contextlib.nullcontext()


def _allocating(stream):
    """Allocations for a launch on `stream`: memory that the allocator hands out for a stream is free of that
    stream's earlier work only, so what a call on another stream than the current one writes is allocated for it."""
    import torch
    return _HERE if stream is None else torch.cuda.stream(stream)


def _opt(t, name, shape, dtypes, device):
    return None if t is None else _want(t, name, shape, dtypes, device)


def _rng_state(rng, device):
    import torch
    return _want(rng, "rng", (2,), (torch.int64, torch.uint64), device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def gtp_layer_norm(x, L: int, w=None, b=None, eps: float = 1e-5, y=None, mean=None, rstd=None, stream=None):
    """(y, mean, rstd): SH features x[N, C, (L+1)^2] normalised by degree (L = 0: the ordinary layer norm over C),
    scaled by w[L+1, C] and, at degree 0, shifted by b[C] (fp32 or None); y has x's type, mean[N] and rstd[N, L+1]
    fp32 are what the backward reads.  y may be x."""
    import torch
    f32 = torch.float32
    if x.dim() != 3 or x.shape[2] != nsh(L):
        raise ValueError("x must be [N, C, (L+1)^2]")
    N, C, _ = x.shape
    dev, one = x.device, (f32,)
    code = _dtype_code(x)
    px = _want(x, "x", x.shape, (x.dtype,))
    pw = _opt(w, "w", (L + 1, C), one, dev)
    pb = _opt(b, "b", (C,), one, dev)
    with _allocating(stream):
        y = torch.empty_like(x) if y is None else y
        mean = torch.empty(N, dtype=f32, device=dev) if mean is None else mean
        rstd = torch.empty((N, L + 1), dtype=f32, device=dev) if rstd is None else rstd
    py = _want(y, "y", x.shape, (x.dtype,), dev)
    pm = _want(mean, "mean", (N,), one, dev)
    pr = _want(rstd, "rstd", (N, L + 1), one, dev)
    _on_gpu(x, "x")
    lib_ = lib()
    _check(lib_.gtp_layer_norm(L, px, code, pw, pb, eps, N, C, py, pm, pr, _stream(stream)), lib_)
    return y, mean, rstd


def gtp_layer_norm_backward(x, dy, L: int, mean, rstd, w=None, need=("dx", "dw", "db"), stream=None):
    """Gradients of <dy, gtp_layer_norm(x, L, w, b)>: a dict with the requested keys among dx (like x), dw[L+1, C] and
    db[C] (fp32); mean, rstd as gtp_layer_norm returned them."""
    import torch
    f32 = torch.float32
    if x.dim() != 3 or x.shape[2] != nsh(L):
        raise ValueError("x must be [N, C, (L+1)^2]")
    unknown = set(need) - {"dx", "dw", "db"}
    if unknown:
        raise ValueError(f"unknown gradients {sorted(unknown)}")
    N, C, _ = x.shape
    dev, one = x.device, (f32,)
    code = _dtype_code(x)
    px = _want(x, "x", x.shape, (x.dtype,))
    pdy = _want(dy, "dy", x.shape, (x.dtype,), dev)
    pw = _opt(w, "w", (L + 1, C), one, dev)
    pm = _want(mean, "mean", (N,), one, dev)
    pr = _want(rstd, "rstd", (N, L + 1), one, dev)
    _on_gpu(x, "x")
    lib_ = lib()
    nbytes = lib_.gtp_layer_norm_backward_work(L, code, N, C) if "dw" in need or "db" in need else 0
    out = {}
    with _allocating(stream):
        if "dx" in need:
            out["dx"] = torch.empty_like(x)
        if "dw" in need:
            out["dw"] = torch.empty((L + 1, C), dtype=f32, device=dev)
        if "db" in need:
            out["db"] = torch.empty(C, dtype=f32, device=dev)
        work = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes > 0 else None
    _check(lib_.gtp_layer_norm_backward(L, px, code, pw, pm, pr, pdy, N, C, _ptr(out.get("dx")), _ptr(out.get("dw")),
                                        _ptr(out.get("db")), _ptr(work), nbytes, _stream(stream)), lib_)
    return out


def gtp_dropout(x, p: float, rng, res=None, y=None, stream=None):
    """y = res + keep x / (1 - p), one draw for each row of x's last dimension (x[..., K]: the K coefficients of a
    channel together; K = 1 drops single values).  rng: int64[2] on the device, (seed, offset), read when the call
    runs; another offset gives other draws.  The gradient is the same call on dy, without res.  y may be x or res."""
    import torch
    if x.dim() < 1:
        raise ValueError("x must have a last dimension")
    code = _dtype_code(x)
    K = x.shape[-1]
    groups = x.numel() // K if K else 0
    dev, own = x.device, (x.dtype,)
    px = _want(x, "x", x.shape, own)
    pres = _opt(res, "res", x.shape, own, dev)
    prng = _rng_state(rng, dev)
    if y is None:
        with _allocating(stream):
            y = torch.empty_like(x)
    py = _want(y, "y", x.shape, own, dev)
    _on_gpu(x, "x")
    lib_ = lib()
    _check(lib_.gtp_dropout(px, pres, code, p, prng, groups, K, py, _stream(stream)), lib_)
    return y


def _attn_rows(t, name, shape, dtype, device):
    """gtp_rows of a [rows, heads, d] tensor whose last dimension is contiguous (a slice of a packed tensor, or an
    expanded input, will do)."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}; expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}; expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}; the other operands are on {device}")
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return t.data_ptr(), row, head


def _attn(q, k, v, scale, q_off, k_off, max_q, max_k, key_mask, p, rng):
    """Validated gtp_attn and the rows of q, k, v, as their fields."""
    import torch
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q must be [Tq, H, d], k and v [Tk, Hk, d]")
    code = _dtype_code(q)
    Tq, H, d = q.shape
    Tk, Hk, _ = k.shape
    dev, dt = q.device, q.dtype
    if H < 1 or Hk < 1 or d < 1 or H % Hk:
        raise ValueError("the number of query heads must be a positive multiple of the number of key heads")
    kshape = (Tk, Hk, d)
    rows = (*_attn_rows(q, "q", q.shape, dt, dev), *_attn_rows(k, "k", kshape, dt, dev),
            *_attn_rows(v, "v", kshape, dt, dev))
    B = None
    for off, name in ((q_off, "q_off"), (k_off, "k_off")):
        if off is None:
            continue
        if off.dim() != 1 or off.shape[0] < 1:
            raise ValueError(f"{name} must be [B + 1]")
        if B is not None and off.shape[0] != B + 1:
            raise ValueError("q_off and k_off must have one length")
        B = off.shape[0] - 1
    if B is None:
        # equal segments: of max_q and max_k rows (a side that has any tells how many), or one of all rows
        B = next((n // most for n, most in ((Tq, max_q), (Tk, max_k)) if n and most), 1)
    max_q = (Tq if q_off is not None else Tq // max(B, 1)) if max_q is None else int(max_q)
    max_k = (Tk if k_off is not None else Tk // max(B, 1)) if max_k is None else int(max_k)
    i64 = (torch.int64,)
    desc = (code, H, Hk, d, B, Tq, Tk, min(max_q, Tq), min(max_k, Tk),
            _opt(q_off, "q_off", (B + 1,), i64, dev) or 0, _opt(k_off, "k_off", (B + 1,), i64, dev) or 0,
            _opt(key_mask, "key_mask", (Tk,), (torch.uint8, torch.bool), dev) or 0,
            1.0 / d ** 0.5 if scale is None else scale, p, 0 if rng is None else _rng_state(rng, dev))
    return desc, rows


def _packed(desc, rows):
    """The structs of a call in one buffer: (buffer, address of gtp_attn, address of each gtp_rows)."""
    n = len(rows) // 3
    buf = ctypes.create_string_buffer(_ATTN.size + ctypes.sizeof(_Rows) * n)
    _ATTN.pack_into(buf, 0, *desc)
    struct.pack_into("<" + _ROWS * n, buf, _ATTN.size, *rows)
    at = ctypes.addressof(buf)
    return buf, at, [at + _ATTN.size + ctypes.sizeof(_Rows) * i for i in range(n)]


def gtp_attention(q, k, v, scale=None, q_off=None, k_off=None, max_q=None, max_k=None, key_mask=None, p: float = 0.0,
                  rng=None, o=None, lse=None, stream=None):
    """(o, lse): softmax attention of q[Tq, H, d] over k, v[Tk, Hk, d] (H a multiple of Hk, d <= 256) within each
    segment (molecule).  q_off, k_off: int64[B+1] device offsets of the segments' rows, max_q and max_k their longest
    (host integers; left out, the whole tensor's length is taken, which costs idle workgroups); without offsets:
    equal segments of max_q and max_k rows, or one.  key_mask[Tk]: 0 = absent key.  scale: 1 / sqrt(d) by default.
    Probabilities are dropped with probability p by the generator state rng (see gtp_dropout).  lse[Tq, H] fp32 is
    what the backward reads.  Tensors may be slices of a packed one (contiguous last dimension)."""
    import torch
    desc, rows = _attn(q, k, v, scale, q_off, k_off, max_q, max_k, key_mask, p, rng)
    dev, shape = q.device, q.shape
    with _allocating(stream):
        o = torch.empty(shape, dtype=q.dtype, device=dev) if o is None else o
        lse = torch.empty(shape[:2], dtype=torch.float32, device=dev) if lse is None else lse
        ro = _attn_rows(o, "o", shape, q.dtype, dev)
        pl = _want(lse, "lse", shape[:2], (torch.float32,), dev)
        _on_gpu(q, "q")
        buf, a, r = _packed(desc, (*rows, *ro))
        lib_ = lib()
        nbytes = lib_.gtp_attention_work(a, 0)
        work = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes > 0 else None
    _check(lib_.gtp_attention(a, *r, pl, _ptr(work), nbytes, _stream(stream)), lib_)
    return o, lse


def gtp_attention_backward(q, k, v, o, do, lse, scale=None, q_off=None, k_off=None, max_q=None, max_k=None,
                           key_mask=None, p: float = 0.0, rng=None, need=("dq", "dk", "dv"), dq=None, dk=None, dv=None,
                           stream=None):
    """Gradients of <do, gtp_attention(q, k, v, ...)[0]>: a dict with the requested keys among dq, dk, dv (dk and dv
    go together).  o, lse as the forward returned them, the other arguments as it had them.  dq, dk, dv: tensors to
    write to (slices of a packed one will do)."""
    import torch
    desc, rows = _attn(q, k, v, scale, q_off, k_off, max_q, max_k, key_mask, p, rng)
    need = set(need)
    if need - {"dq", "dk", "dv"}:
        raise ValueError(f"unknown gradients {sorted(need - {'dq', 'dk', 'dv'})}")
    dev, dt, qs, ks = q.device, q.dtype, q.shape, k.shape
    ro = _attn_rows(o, "o", qs, dt, dev)
    rdo = _attn_rows(do, "do", qs, dt, dev)
    pl = _want(lse, "lse", qs[:2], (torch.float32,), dev)
    keys = "dk" in need or "dv" in need
    none = (0, 0, 0)
    with _allocating(stream):
        out = {}
        if "dq" in need:
            out["dq"] = torch.empty(qs, dtype=dt, device=dev) if dq is None else dq
        if keys:
            out["dk"] = torch.empty(ks, dtype=dt, device=dev) if dk is None else dk
            out["dv"] = torch.empty(ks, dtype=dt, device=dev) if dv is None else dv
        rdq = _attn_rows(out["dq"], "dq", qs, dt, dev) if "dq" in need else none
        rdk = _attn_rows(out["dk"], "dk", ks, dt, dev) if keys else none
        rdv = _attn_rows(out["dv"], "dv", ks, dt, dev) if keys else none
        _on_gpu(q, "q")
        buf, a, r = _packed(desc, (*rows, *ro, *rdo, *rdq, *rdk, *rdv))
        lib_ = lib()
        nbytes = lib_.gtp_attention_work(a, 1)
        work = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes > 0 else None
    _check(lib_.gtp_attention_backward(a, *r[:5], pl, r[5] if "dq" in need else None, *(r[6:] if keys else (None, None)),
                                       _ptr(work), nbytes, _stream(stream)), lib_)
    return {n: t for n, t in out.items() if n in need}


def gtp_stream_probe(mode: int, src, dst, stream=None):
    """HBM streaming probe: mode 0 reads src (dst: >= 1 float), 1 writes dst, 2 copies src to dst,
    3 writes the sum of src's two halves to dst (>= half of src)."""
    nbytes = (dst if mode == 1 else src).numel() * (dst if mode == 1 else src).element_size()
    if mode == 2 and dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst smaller than src")
    if mode == 3 and dst.numel() * dst.element_size() < nbytes // 2:
        raise ValueError("dst smaller than half of src")
    sp = ctypes.c_void_p(None) if mode == 1 else ctypes.c_void_p(src.data_ptr())
    _check(lib().gtp_stream_probe(mode, sp, ctypes.c_void_p(dst.data_ptr()), nbytes, _stream(stream)))


def gtp_compute_probe(mode: int, iters: int, sink, stream=None) -> float:
    """fp32 compute probe: mode 0 VALU FMA chains, 1 MFMA chains; returns the flops launched."""
    ps = _want(sink, "sink", (1,), _f32())
    fl = ctypes.c_double(0.0)
    _check(lib().gtp_compute_probe(mode, iters, ps, ctypes.byref(fl), _stream(stream)))
    return fl.value


def gtp_debug_host_pipeline(plan: Plan, x1, x2):
    """fp64 host evaluation of the plan's sampled pipeline (table check only)."""
    import numpy as np
    a = np.ascontiguousarray(x1, dtype=np.float64).reshape(-1, nsh(plan.L1))
    b = np.ascontiguousarray(x2, dtype=np.float64).reshape(-1, nsh(plan.L2))
    y = np.zeros((a.shape[0], nsh(plan.Lout)), dtype=np.float64)
    _check(plan.lib.gtp_debug_host_pipeline(plan.handle, a.ctypes.data_as(_DP), b.ctypes.data_as(_DP), a.shape[0],
                                            y.ctypes.data_as(_DP)), plan.lib)
    return y
