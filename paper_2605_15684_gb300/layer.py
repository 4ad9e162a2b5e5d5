"""A layer around its attention (include/ssba.h, same names): the root-mean-square norm, products with weights
and what follows them, the gated half of a feed-forward block, rotary positions with several axes, and
the gradients of each.

Argument marshalling only, as in api.py: tensors are checked, outputs and workspaces allocated on the call's
stream, and every step runs in the library's kernels on the current device. Calls on the current stream that leave
their outputs to be allocated take a native short way (csrc/host/layer_call.cpp).

    y, h, rstd = rms_norm(x, w, residual=r)            # h = x + r, y = its norm
    q, s, h, rstd = rms_norm(x, w, residual=r, e4m3=True)
    z = linear(q, W8, x_scale=s, w_scale=ws, bias=b)   # e4m3 rows and weights
    a = gated_linear(y, Wgu)                           # act(y Wg^T) * (y Wu^T)
    x = linear(a, Wd, residual=h)
    rope_axes(qkv[:, :, 0], pos, (16, 24, 24), out=Q.transpose(1, 2))
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

import torch

from . import api, build
from .api import (SSBA_BF16, SSBA_ERR_INVALID, SSBA_FP32, SsbaError, _check, _empty, _out, _raise_on, _side,
                  _lock, _stream_ptr, load_library)

SSBA_E4M3 = 2
E4M3 = torch.float8_e4m3fn
ACTS = {None: 0, "relu": 1, "gelu": 2, "silu": 3}
ROPE_LAYOUTS = {"pairs": 0, "halves": 1}
ROPE_MAX_AXES = 4
_I32 = 2 ** 31


class _LinearDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "N", "K", "dtype", "act", "gated")]


class _RopeDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("axes", ctypes.c_int32), ("sections", ctypes.c_int32 * ROPE_MAX_AXES), ("layout", ctypes.c_int32),
                ("shared", ctypes.c_int32), ("inverse", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("base", ctypes.c_double)]


_ext = None


def _extension():
    """The native short way into the calls (csrc/host/layer_call.cpp), made by build() beside the library."""
    global _ext
    lib = load_library()
    with _lock:
        if _ext is None:
            path = build.call_file("layer_call")
            if not os.path.exists(path):
                raise SsbaError(api.SSBA_ERR_CUDA, f"{path} is missing: run paper_2605_15684_gb300.build.build()")
            spec = importlib.util.spec_from_file_location("_layer_call", path)
            ext = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(ext)
            ext.bind(*(ctypes.cast(getattr(lib, "ssba_" + n), ctypes.c_void_p).value
                       for n in ("rms_norm", "rms_norm_backward", "rms_norm_backward_workspace_bytes", "linear", "linear_backward",
                                 "linear_backward_workspace_bytes", "rope_axes")))
            _ext = ext
    return _ext


def _invalid(msg: str):
    raise SsbaError(SSBA_ERR_INVALID, msg)


def _sized(n: int, name: str) -> int:
    if n >= _I32:
        _invalid(f"{name}={n} is too large")
    return n


def _matrix(t, name: str, dtypes):
    """A 2-D contiguous CUDA tensor on the current device, of one of ``dtypes``; returns its shape."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        _invalid(f"{name} must be a 2-D tensor")
    if t.dtype not in dtypes:
        _invalid(f"{name} has dtype {t.dtype}, expected one of {', '.join(str(d) for d in dtypes)}")
    _check(t, name, t.shape, t.dtype)
    if t.device.index != torch.cuda.current_device():
        _invalid(f"{name} lies on {t.device}, which is not the current device")
    _sized(t.shape[0], f"{name}.shape[0]")
    _sized(t.shape[1], f"{name}.shape[1]")
    return t.shape


def _with(t, name: str, shape, dtype, dev):
    """Another input of the call: None, or a checked tensor on the same device."""
    if t is None:
        return None
    _check(t, name, shape, dtype)
    if t.device != dev:
        _invalid(f"{name} lies on {t.device}, the call's other tensors on {dev}")
    return t.data_ptr()


def _result(t, name: str, shape, dtype, dev, side):
    if t is not None and isinstance(t, torch.Tensor) and t.is_cuda and t.device != dev:
        _invalid(f"{name} lies on {t.device}, the call's other tensors on {dev}")
    return _out(t, name, shape, dtype, dev, side)


def _workspace(ws, need: int, dev, side):
    if ws is None:
        ws = _empty((max(need, 16),), torch.uint8, dev, side, scratch=True)
    elif isinstance(ws, torch.Tensor) and ws.is_cuda and ws.device != dev:
        _invalid(f"workspace lies on {ws.device}, the call's other tensors on {dev}")
    return ws, *api._ws_args(ws)


def _act(act, gated: bool = False) -> int:
    if act not in ACTS or (gated and act is None):
        _invalid(f"act={act!r}: one of {', '.join(repr(a) for a in ACTS if a or not gated)}")
    return ACTS[act]


_NORM_TYPES = (torch.bfloat16, torch.float32)


def rms_norm(x, w, residual=None, eps: float = 1e-6, e4m3: bool = False, y=None, scale=None, h=None, rstd=None,
             stream=None):
    """ssba_rms_norm: x [T, D] bf16 or fp32, w [D] fp32 -> (y, h, rstd), or with e4m3 (y, scale, h, rstd): h = x +
    residual (x itself without one), y its norm times w (e4m3: values whose rows stand for themselves times scale [T], a power
    of two), rstd [T] fp32 for rms_norm_backward. ``h`` may be x or residual, ``y`` (not e4m3) may be x."""
    if stream is None and y is None and h is None and rstd is None and scale is None:
        out = (_ext or _extension()).rms_norm(x, w, residual, eps, e4m3)
        if out.__class__ is tuple:
            return out
        if out is not None:
            _raise_on(out)
    lib = load_library()
    T, D = _matrix(x, "x", _NORM_TYPES)
    dt, dev = x.dtype, x.device
    wp, rp = _with(w, "w", (D,), torch.float32, dev), _with(residual, "residual", x.shape, dt, dev)
    if wp is None:
        _invalid("w must be a torch.Tensor")
    if not e4m3 and scale is not None or residual is None and h is not None:
        _invalid("scale is an output with e4m3, and h with a residual")
    side = _side(stream, dev)
    y = _result(y, "y", x.shape, E4M3 if e4m3 else dt, dev, side)
    if e4m3:
        scale = _result(scale, "scale", (T,), torch.float32, dev, side)
    if residual is not None:
        h = _result(h, "h", x.shape, dt, dev, side)
    rstd = _result(rstd, "rstd", (T,), torch.float32, dev, side)
    rc = lib.ssba_rms_norm(x.data_ptr(), rp, wp, T, D, SSBA_BF16 if dt is torch.bfloat16 else SSBA_FP32, eps,
                           h.data_ptr() if residual is not None else None, y.data_ptr(), scale.data_ptr() if e4m3 else None,
                           rstd.data_ptr(), _stream_ptr(stream))
    if rc:
        _raise_on(rc)
    h = x if residual is None else h
    return (y, scale, h, rstd) if e4m3 else (y, h, rstd)


def rms_norm_backward_workspace_bytes(T: int, D: int, dtype=torch.bfloat16) -> int:
    if dtype not in _NORM_TYPES:
        _invalid(f"unsupported dtype {dtype}")
    return int(load_library().ssba_rms_norm_backward_workspace_bytes(_sized(T, "T"), _sized(D, "D"),
                                                                     SSBA_BF16 if dtype == torch.bfloat16 else SSBA_FP32))


def rms_norm_backward(dy, h, w, rstd, dh=None, dx=None, dw=None, workspace=None, stream=None):
    """ssba_rms_norm_backward: dy, and the h (or x) and rstd of the forward call -> (dx [T, D], dw [D] fp32); dx is the
    gradient of x and of the residual alike, with ``dh``, which reaches h from elsewhere, added. ``dx`` may be dy or dh."""
    if stream is None and dx is None and dw is None and workspace is None:
        out = (_ext or _extension()).rms_norm_backward(dy, h, w, rstd, dh)
        if out.__class__ is tuple:
            return out
        if out is not None:
            _raise_on(out)
    lib = load_library()
    T, D = _matrix(h, "h", _NORM_TYPES)
    dt, dev = h.dtype, h.device
    code = SSBA_BF16 if dt is torch.bfloat16 else SSBA_FP32
    dyp, dhp = _with(dy, "dy", h.shape, dt, dev), _with(dh, "dh", h.shape, dt, dev)
    wp, kp = _with(w, "w", (D,), torch.float32, dev), _with(rstd, "rstd", (T,), torch.float32, dev)
    if dyp is None or wp is None or kp is None:
        _invalid("dy, w and rstd must be torch.Tensors")
    side = _side(stream, dev)
    dx = _result(dx, "dx", h.shape, dt, dev, side)
    dw = _result(dw, "dw", (D,), torch.float32, dev, side)
    need = int(lib.ssba_rms_norm_backward_workspace_bytes(T, D, code)) if workspace is None else 0
    workspace, sp, sn = _workspace(workspace, need, dev, side)
    rc = lib.ssba_rms_norm_backward(dyp, h.data_ptr(), wp, kp, dhp, T, D, code, dx.data_ptr(), dw.data_ptr(), sp, sn,
                                    _stream_ptr(stream))
    if rc:
        _raise_on(rc)
    return dx, dw


def _product(x, W, bias, residual, act, x_scale, w_scale, pre, y, z, stream, gated):
    if stream is None and y is None and z is None:
        out = (_ext or _extension()).linear(x, W, bias, residual, x_scale, w_scale, _act(act, gated), pre, gated)
        if out.__class__ is int:
            _raise_on(out)
        if out is not None:
            return out
    lib = load_library()
    T, K = _matrix(x, "x", (torch.bfloat16, E4M3))
    rows, k = _matrix(W, "W", (x.dtype,))
    dev = x.device
    if k != K or (gated and rows % 2):
        _invalid(f"W has shape {tuple(W.shape)}, expected [{'2 N' if gated else 'N'}, {K}]")
    if W.device != dev:
        _invalid(f"W lies on {W.device}, the call's other tensors on {dev}")
    N = rows // 2 if gated else rows
    f8 = x.dtype is E4M3
    if (x_scale is not None) != f8 or (w_scale is not None) != f8:
        _invalid("x_scale and w_scale are given for e4m3 rows and weights, and for nothing else")
    xs, ws = _with(x_scale, "x_scale", (T,), torch.float32, dev), _with(w_scale, "w_scale", (rows,), torch.float32, dev)
    bp, rp = _with(bias, "bias", (N,), torch.float32, dev), _with(residual, "residual", (T, N), torch.bfloat16, dev)
    d = _LinearDesc(T, N, K, SSBA_E4M3 if f8 else SSBA_BF16, _act(act, gated), gated)
    side = _side(stream, dev)
    y = _result(y, "y", (T, N), torch.bfloat16, dev, side)
    keep = pre or z is not None
    if keep:
        z = _result(z, "z", (T, rows), torch.bfloat16, dev, side)
    rc = lib.ssba_linear(ctypes.byref(d), x.data_ptr(), W.data_ptr(), xs, ws, bp, rp, y.data_ptr(),
                         z.data_ptr() if keep else None, _stream_ptr(stream))
    if rc:
        _raise_on(rc)
    return (y, z) if keep else y


def linear(x, W, bias=None, residual=None, act=None, x_scale=None, w_scale=None, pre: bool = False, y=None, z=None,
           stream=None):
    """ssba_linear: y = act(z) + residual with z = x W^T (x_scale w_scale) + bias; x [T, K], W [N, K] bf16, or both e4m3
    with fp32 scales [T] and [N] (rms_norm makes such rows; of weights once: s = 2 ** ceil(log2(max |W_n| / 448)), W / s
    rounded); bias [N] fp32, residual [T, N] bf16 (may be ``y``); act None, "relu", "gelu" (its tanh form, which is not torch's default) or "silu".
    Returns y [T, N] bf16, or with ``pre`` (y, z): z is what linear_backward needs of an activation."""
    return _product(x, W, bias, residual, act, x_scale, w_scale, pre, y, z, stream, 0)


def gated_linear(x, W, act="silu", x_scale=None, w_scale=None, pre: bool = False, y=None, z=None, stream=None):
    """ssba_linear, gated: y = act(x Wg^T) * (x Wu^T), W [2 F, K] the rows of Wg, then those of Wu; types and act ("gelu" is its
    tanh form) as linear.
    Returns y [T, F] bf16, or with ``pre`` (y, z [T, 2 F]): both products, which gated_linear_backward needs."""
    return _product(x, W, None, None, act, x_scale, w_scale, pre, y, z, stream, 1)


def test_linear_timeout(x, W, y, gated: bool = False, budget_ns: int = 2_000_000, stream=None) -> None:
    """ssba_test_linear_timeout: the products' failure-detection test hook (include/ssba.h)."""
    lib = load_library()
    T, K = _matrix(x, "x", (torch.bfloat16,))
    rows, _ = _matrix(W, "W", (torch.bfloat16,))
    N = rows // 2 if gated else rows
    _check(W, "W", (rows, K), torch.bfloat16)
    _check(y, "y", (T, N), torch.bfloat16)
    d = _LinearDesc(T, N, K, SSBA_BF16, _act("silu" if gated else None), int(gated))
    _raise_on(lib.ssba_test_linear_timeout(ctypes.byref(d), x.data_ptr(), W.data_ptr(), y.data_ptr(), int(budget_ns),
                                           _stream_ptr(stream)))


def _linear_desc_of(T, N, K, act, gated):
    return _LinearDesc(_sized(T, "T"), _sized(N, "N"), _sized(K, "K"), SSBA_BF16, _act(act, gated), gated)


def linear_backward_workspace_bytes(T: int, N: int, K: int, act=None, gated: bool = False) -> int:
    d = _linear_desc_of(T, N, K, act, int(gated))
    return int(load_library().ssba_linear_backward_workspace_bytes(ctypes.byref(d)))


def _product_backward(dy, x, W, z, act, db, dx, dW, workspace, stream, gated, bias):
    if stream is None and db is None and workspace is None and (dx is None or dx is False) and (dW is None or dW is False):
        out = (_ext or _extension()).linear_backward(dy, x, W, z if act is not None else None, _act(act, gated), gated, bias,
                                                     dx is None, dW is None)
        if out.__class__ is tuple:
            return out
        if out is not None:
            _raise_on(out)
    lib = load_library()
    bf = torch.bfloat16
    T, N = _matrix(dy, "dy", (bf,))
    dev = dy.device
    if dx is False and dW is False and not bias:
        _invalid("nothing to compute: dx and dW are both False")
    rows = 2 * N if gated else N
    if dx is False and dW is False:
        K = x.shape[1] if isinstance(x, torch.Tensor) and x.dim() == 2 else 16
    else:
        K = _matrix(W if dx is not False else x, "W" if dx is not False else "x", (bf,))[1]
    xp = _with(x, "x", (T, K), bf, dev) if dW is not False else None
    Wp = _with(W, "W", (rows, K), bf, dev) if dx is not False else None
    if dW is not False and xp is None:
        _invalid("x must be a torch.Tensor")
    code = _act(act, gated)
    if code and z is None:
        _invalid("z, kept by the forward call, is needed with an activation")
    zp = _with(z, "z", (T, rows), bf, dev) if code else None
    d = _LinearDesc(T, N, K, SSBA_BF16, code, gated)
    side = _side(stream, dev)
    dx = None if dx is False else _result(dx, "dx", (T, K), bf, dev, side)
    dW = None if dW is False else _result(dW, "dW", (rows, K), bf, dev, side)
    db = _result(db, "db", (N,), torch.float32, dev, side) if bias else None
    need = int(lib.ssba_linear_backward_workspace_bytes(ctypes.byref(d))) if workspace is None else 0
    workspace, sp, sn = _workspace(workspace, need, dev, side)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    rc = lib.ssba_linear_backward(ctypes.byref(d), dy.data_ptr(), xp, Wp, zp, ptr(dx), ptr(dW), ptr(db), sp, sn,
                                  _stream_ptr(stream))
    if rc:
        _raise_on(rc)
    return dx, dW, db


def linear_backward(dy, x, W, z=None, act=None, bias: bool = False, dx=None, dW=None, db=None, workspace=None,
                    stream=None):
    """ssba_linear_backward: (dx [T, K] bf16, dW [N, K] bf16, db [N] fp32 or None) for the gradient dy [T, N] of y, which is
    the residual's own as it is. ``bias``: db is wanted. dx=False or dW=False leaves that one out (None); z is
    the forward call's, with an activation."""
    return _product_backward(dy, x, W, z, act, db, dx, dW, workspace, stream, 0, bias or db is not None)


def gated_linear_backward(dy, x, W, z, act="silu", dx=None, dW=None, workspace=None, stream=None):
    """ssba_linear_backward, gated: (dx [T, K], dW [2 F, K]) bf16 for the gradient dy [T, F] and the forward call's z."""
    return _product_backward(dy, x, W, z, act, None, dx, dW, workspace, stream, 1, False)[:2]


def _heads(t, name: str, dtypes):
    """[B, T, heads, d] or [T, heads, d] with the last dimension side by side -> its 4-D shape and three strides."""
    if not isinstance(t, torch.Tensor) or t.dim() not in (3, 4):
        _invalid(f"{name} must be a tensor [B, T, heads, d] or [T, heads, d]")
    if not t.is_cuda:
        _invalid(f"{name} must be a CUDA tensor (got {t.device})")
    if t.dtype not in dtypes:
        _invalid(f"{name} has dtype {t.dtype}, expected one of {', '.join(str(d) for d in dtypes)}")
    if t.shape[-1] != 1 and t.stride(-1) != 1:
        _invalid(f"{name}'s last dimension must be contiguous")
    s, st = t.shape, t.stride()
    return ((1, *s), (0, *st)) if t.dim() == 3 else (tuple(s), st)


def _dense_heads(shape, strides) -> bool:
    """Whether no two elements share an address: sorted by stride, each dimension steps past those inside it."""
    reach = 1
    for st, n in sorted((st, n) for n, st in zip(shape, (*strides[:3], 1)) if n > 1):
        if st < reach:
            return False
        reach = st * (n - 1) + reach
    return True


_rope_descs: dict = {}


def _rope_desc(key):
    """The C struct of a call's sizes and rule, kept by its values (a model's layers share a few); no tensor is kept."""
    d = _rope_descs.get(key)
    if d is None:
        B, T, H, D, axes, layout, shared, inverse, dt, base = key
        if layout not in ROPE_LAYOUTS:
            _invalid(f"layout={layout!r}: 'pairs' or 'halves'")
        if not 1 <= len(axes) <= ROPE_MAX_AXES:
            _invalid(f"axes must be the pairs of 1..{ROPE_MAX_AXES} axes")
        if any(not 0 < a < 65536 for a in axes):
            _invalid("every axis has at least one pair")
        for n, v in (("B", B), ("T", T), ("heads", H), ("head_dim", D)):
            _sized(v, n)
        d = _RopeDesc(B, T, H, D, len(axes), (ctypes.c_int32 * ROPE_MAX_AXES)(*axes), ROPE_LAYOUTS[layout], shared, inverse,
                      SSBA_BF16 if dt is torch.bfloat16 else SSBA_FP32, base)
        if len(_rope_descs) >= 256:
            _rope_descs.clear()
        _rope_descs[key] = d
    return d


def rope_axes(x, positions, axes, base: float = 10000.0, layout: str = "pairs", shared: bool = False,
              inverse: bool = False, out=None, stream=None):
    """ssba_rope_axes: x [B, T, heads, d] (or [T, heads, d]) bf16 or fp32, any strides with the last dimension side by
    side, turned by positions [T, A] or [B, T, A] int32; axes: the pairs of each of the A axes, 2 sum(axes) <= d, dimensions
    behind them as they were. layout "pairs" (2j, 2j + 1) or "halves" (j, j + sum(axes)); shared False: each axis has the whole range
    of rates, True: the pairs share one. inverse: by the negative angles, which gives the gradient. ``out``: of
    x's shape at any strides; x itself for in place. Returns out."""
    if stream is None and layout in ROPE_LAYOUTS:
        got = (_ext or _extension()).rope(x, positions, axes, base, ROPE_LAYOUTS[layout], shared, inverse, out)
        if got.__class__ is int:
            _raise_on(got)
        if got is not None:
            return got
    lib = load_library()
    shape, xs = _heads(x, "x", _NORM_TYPES)
    B, T, H, D = shape
    dev = x.device
    if dev.index != torch.cuda.current_device():
        _invalid(f"x lies on {dev}, which is not the current device")
    axes = tuple(int(a) for a in axes)
    A = len(axes)
    if not isinstance(positions, torch.Tensor) or positions.dim() not in (2, 3):
        _invalid("positions must be a tensor [T, A] or [B, T, A]")
    each = positions.dim() == 3
    pp = _with(positions, "positions", (B, T, A) if each else (T, A), torch.int32, dev)
    d = _rope_desc((B, T, H, D, axes, layout, bool(shared), bool(inverse), x.dtype, float(base)))
    if out is None:
        out = _empty(x.shape, x.dtype, dev, _side(stream, dev))
    oshape, os = _heads(out, "out", (x.dtype,))
    if oshape != shape or out.dim() != x.dim():
        _invalid(f"out has shape {tuple(out.shape)}, expected {tuple(x.shape)}")
    if out.device != dev:
        _invalid(f"out lies on {out.device}, the call's other tensors on {dev}")
    if not _dense_heads(shape, os):
        _invalid("elements of out may not share an address")
    rc = lib.ssba_rope_axes(ctypes.byref(d), x.data_ptr(), (ctypes.c_int64 * 3)(*xs[:3]), pp, T * A if each else 0,
                            out.data_ptr(), (ctypes.c_int64 * 3)(*os[:3]), _stream_ptr(stream))
    if rc:
        _raise_on(rc)
    return out
