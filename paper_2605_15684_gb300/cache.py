"""Binding of the paged 8-bit K/V cache (``ssba_cache_*`` in include/ssba.h), and the host's side of it:
which pages hold which sequence.

``cache_append``, ``cache_select``, ``cache_attend`` and ``cache_copy`` marshal arguments as api.py does
(device, dtype, shape, contiguity; the current stream unless ``stream`` is given). ``PagedCache`` owns a
pool, keeps a page table with reference counts, and makes those calls for sequences by their ids: append,
attend, fork with copy on write, free, compact. It holds integers only; every byte of the cache is moved by
the library's kernels.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import api
from .api import (SSBA_BF16, SSBA_ERR_INVALID, SSBA_ERR_WORKSPACE, SSBA_FP32, SsbaError, _check, _empty, _lock,
                  _raise_on, _side, _stream_ptr, load_library)

PAGE = 64
_TICKET_BYTES = 4096  # of the attention's workspace, zero between calls (SSBA_CACHE_TICKET_BYTES)
_E4M3 = torch.float8_e4m3fn


@dataclass
class CacheDesc:
    """Python mirror of ``ssba_cache_desc``."""
    heads: int
    kv_heads: int
    head_dim: int
    pages: int
    dtype: torch.dtype = torch.bfloat16
    softmax_scale: float = 0.0

    def c(self) -> api._CacheDesc:
        if self.dtype == torch.bfloat16:
            dt = SSBA_BF16
        elif self.dtype == torch.float32:
            dt = SSBA_FP32
        else:
            raise SsbaError(SSBA_ERR_INVALID, f"unsupported dtype {self.dtype}")
        return api._CacheDesc(self.heads, self.kv_heads, self.head_dim, self.pages, dt, float(self.softmax_scale))


class Cache:
    """The pool's tensors: K, V float8_e4m3fn [pages, kv_heads, 64, head_dim]; k_scale, v_scale fp32
    [pages, kv_heads]; k_mean fp32 [pages, kv_heads, head_dim]. They are checked here, once, and are the pool's
    for good: a tensor may not be resized or given other memory while the calls use it."""
    __slots__ = ("K", "V", "k_scale", "v_scale", "k_mean", "_shape", "_dev", "_ref", "_c")

    def __init__(self, K: torch.Tensor, V: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                 k_mean: torch.Tensor):
        if not isinstance(K, torch.Tensor) or K.dim() != 4 or K.shape[2] != PAGE:
            raise SsbaError(SSBA_ERR_INVALID, f"K must be a tensor [pages, kv_heads, {PAGE}, head_dim]")
        pages, kv, _, d = K.shape
        tensors = (K, V, k_scale, v_scale, k_mean)
        for t, n, shape, dtype in ((K, "K", K.shape, _E4M3), (V, "V", K.shape, _E4M3),
                                   (k_scale, "k_scale", (pages, kv), torch.float32),
                                   (v_scale, "v_scale", (pages, kv), torch.float32),
                                   (k_mean, "k_mean", (pages, kv, d), torch.float32)):
            _check(t, "cache." + n, shape, dtype)
            if t.device != K.device:
                raise SsbaError(SSBA_ERR_INVALID, f"cache.{n} is on {t.device}, K on {K.device}")
        put = object.__setattr__
        for n, t in zip(Cache.__slots__, tensors):
            put(self, n, t)
        put(self, "_shape", (pages, kv, d))
        put(self, "_dev", K.device)
        c = api._Cache(*(t.data_ptr() for t in tensors))
        put(self, "_c", c)
        put(self, "_ref", ctypes.byref(c))

    def __setattr__(self, name, value):
        raise AttributeError("a cache's tensors are given when it is made")


class _Plan:
    """What the calls derive from a descriptor's values alone: the C struct and the sizes."""
    __slots__ = ("c", "ref", "dtype", "heads", "kv", "d", "shape")

    def __init__(self, desc: CacheDesc, c):
        self.c, self.ref, self.dtype = c, ctypes.byref(c), desc.dtype
        self.heads, self.kv, self.d = desc.heads, desc.kv_heads, desc.head_dim
        self.shape = (desc.pages, desc.kv_heads, desc.head_dim)


_plans: dict = {}


def _plan(desc: CacheDesc) -> _Plan:
    """The plan of a descriptor, kept by its values."""
    key = (desc.heads, desc.kv_heads, desc.head_dim, desc.pages, desc.dtype, desc.softmax_scale)
    pl = _plans.get(key)
    if pl is None:
        if min(key[:4]) <= 0 or max(key[:4]) > 2 ** 31 - 1:  # the struct keeps 32 bits
            raise SsbaError(SSBA_ERR_INVALID, f"sizes must be positive and below 2^31: {desc}")
        pl = _Plan(desc, desc.c())
        if len(_plans) >= api._PLAN_CAP:
            _plans.clear()
        _plans[key] = pl
    return pl


def _pool(pl: _Plan, cache: Cache):
    """The device of a pool of the plan's sizes; it has to be the current one, where kernels run."""
    if not isinstance(cache, Cache):
        raise SsbaError(SSBA_ERR_INVALID, "cache must be a Cache")
    if cache._shape != pl.shape:
        raise SsbaError(SSBA_ERR_INVALID, f"cache of (pages, kv_heads, head_dim) {cache._shape}, expected {pl.shape}")
    dev = cache._dev
    if dev.index != torch._C._cuda_getDevice():
        raise SsbaError(SSBA_ERR_INVALID, f"the cache is on {dev}, the current device is cuda:{torch.cuda.current_device()}")
    return dev


def _on(t, name: str, shape, dtype, dev) -> None:
    """_check, and that the tensor is on the call's device."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev.index
            and t.is_contiguous()):
        return
    _check(t, name, shape, dtype)
    raise SsbaError(SSBA_ERR_INVALID, f"{name} is on {t.device}, the cache on {dev}")


def _rows(x, name: str, heads: int, pl: _Plan, dev) -> int:
    """Rows of a [T, heads, head_dim] tensor."""
    T = x.shape[0] if isinstance(x, torch.Tensor) and x.dim() == 3 else 0
    _on(x, name, (T, heads, pl.d), pl.dtype, dev)
    return T


def _batch(table, lens, cu, dev):
    """(table, width, lens, cu, B) as the C calls take them."""
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise SsbaError(SSBA_ERR_INVALID, "table must be a 2-D tensor [B, width]")
    shape = table.shape
    B, width = shape
    _on(table, "table", shape, torch.int32, dev)
    _on(lens, "lens", (B,), torch.int32, dev)
    _on(cu, "cu", (B + 1,), torch.int32, dev)
    return table.data_ptr(), width, lens.data_ptr(), cu.data_ptr(), B


def _result(t, name: str, shape, dtype, dev, side):
    """An output: allocated when the caller gave none, else checked."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev) if side is None else _empty(shape, dtype, dev, side)
    _on(t, name, shape, dtype, dev)
    return t


def cache_alloc(desc: CacheDesc, device="cuda") -> Cache:
    """A pool of desc.pages pages (contents undefined: an append writes what later calls read)."""
    pages, kv, d = _plan(desc).shape
    kw = dict(device=device, dtype=torch.float32)
    return Cache(*(torch.empty((pages, kv, PAGE, d), device=device, dtype=_E4M3) for _ in range(2)),
                 *(torch.empty((pages, kv), **kw) for _ in range(2)), torch.empty((pages, kv, d), **kw))


def cache_append(desc: CacheDesc, cache: Cache, k, v, table, lens, cu, stream=None) -> Cache:
    """ssba_cache_append: k, v [T, kv_heads, head_dim] into the pages of their sequences; table [B, width],
    lens [B] (tokens held before), cu [B + 1], all int32. Returns the cache."""
    lib = api._lib or load_library()
    pl = _plan(desc)
    dev = _pool(pl, cache)
    T = _rows(k, "k", pl.kv, pl, dev)
    _on(v, "v", k.shape, pl.dtype, dev)
    batch = _batch(table, lens, cu, dev)
    _raise_on(lib.ssba_cache_append(pl.ref, cache._ref, k.data_ptr(), v.data_ptr(), T, *batch,
                                    _stream_ptr(stream)))
    return cache


def cache_select(desc: CacheDesc, cache: Cache, q, table, lens, cu, keep: int, first: int = 1, idx=None, cnt=None,
                 stream=None):
    """ssba_cache_select: q [T, heads, head_dim] -> (idx [T, kv_heads, keep], cnt [T, kv_heads]) int32.
    lens: tokens held, the rows of q among them."""
    lib = api._lib or load_library()
    pl = _plan(desc)
    dev = _pool(pl, cache)
    T = _rows(q, "q", pl.heads, pl, dev)
    batch = _batch(table, lens, cu, dev)
    if not 0 <= first < keep:
        raise SsbaError(SSBA_ERR_INVALID, f"keep={keep} must be more than first={first}, first >= 0")
    side = _side(stream, dev)
    idx = _result(idx, "idx", (T, pl.kv, keep), torch.int32, dev, side)
    cnt = _result(cnt, "cnt", (T, pl.kv), torch.int32, dev, side)
    _raise_on(lib.ssba_cache_select(pl.ref, cache._ref, q.data_ptr(), T, *batch, keep, first, idx.data_ptr(),
                                    cnt.data_ptr(), _stream_ptr(stream)))
    return idx, cnt


def cache_attend_workspace_bytes(desc: CacheDesc) -> int:
    lib = load_library()
    n = int(lib.ssba_cache_attend_workspace_bytes(_plan(desc).ref))
    if n == 0:
        _raise_on(SSBA_ERR_INVALID)
    return n


_ws: dict = {}
_ws_need: dict = {}  # per device: the same for every descriptor


def _default_workspace(pl: _Plan, lib, dev, stream, side):
    """A workspace kept per (device, stream): the calls of one stream run in order and can share it. A capture
    gets one of its own, so that no two graphs, and no graph and an eager call, meet in one."""
    need = _ws_need.get(dev.index)
    if need is None:
        need = int(lib.ssba_cache_attend_workspace_bytes(pl.ref))
        if need == 0:
            _raise_on(SSBA_ERR_INVALID)
        _ws_need[dev.index] = need
    if side is None and not torch.cuda.is_current_stream_capturing():
        key = (dev.index, torch._C._cuda_getCurrentRawStream(dev.index))
        ws = _ws.get(key)
        if ws is not None:
            return ws
    with torch.cuda.stream(side):  # allocated and filled on the stream that uses it
        if torch.cuda.is_current_stream_capturing():
            # the fill is a node of the graph, so no later call may count on it
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
            ws[:_TICKET_BYTES].zero_()
            return ws
        key = (dev.index, torch._C._cuda_getCurrentRawStream(dev.index))
        with _lock:
            ws = _ws.get(key)
            if ws is None:
                ws = _ws[key] = torch.zeros(need, dtype=torch.uint8, device=dev)
    return ws


def cache_attend(desc: CacheDesc, cache: Cache, q, table, lens, cu, idx=None, cnt=None, O=None, lse=None,
                 workspace="default", stream=None):
    """ssba_cache_attend: q [T, heads, head_dim] -> (O [T, heads, head_dim], lse [T, heads] fp32), over every
    page of the rows' sequences, or over the lists (idx, cnt) of cache_select."""
    lib = api._lib or load_library()
    pl = _plan(desc)
    dev = _pool(pl, cache)
    T = _rows(q, "q", pl.heads, pl, dev)
    batch = _batch(table, lens, cu, dev)
    keep = 0
    if (idx is None) != (cnt is None):
        raise SsbaError(SSBA_ERR_INVALID, "idx and cnt come together")
    if idx is not None:
        keep = int(idx.shape[2]) if isinstance(idx, torch.Tensor) and idx.dim() == 3 else 0
        _on(idx, "idx", (T, pl.kv, keep), torch.int32, dev)
        _on(cnt, "cnt", (T, pl.kv), torch.int32, dev)
    side = _side(stream, dev)
    O = _result(O, "O", q.shape, pl.dtype, dev, side)
    lse = _result(lse, "lse", (T, pl.heads), torch.float32, dev, side)
    if isinstance(workspace, str):
        workspace = _default_workspace(pl, lib, dev, stream, side)
    elif workspace is None:
        raise SsbaError(SSBA_ERR_WORKSPACE, "cache_attend needs a workspace")
    wp, wn = api._ws_args(workspace)
    _raise_on(lib.ssba_cache_attend(pl.ref, cache._ref, q.data_ptr(), T, *batch,
                                    idx.data_ptr() if idx is not None else None,
                                    cnt.data_ptr() if cnt is not None else None, keep, O.data_ptr(), lse.data_ptr(),
                                    wp, wn, _stream_ptr(stream)))
    return O, lse


def cache_copy(desc: CacheDesc, cache: Cache, src, dst, stream=None) -> Cache:
    """ssba_cache_copy: pages src[i] -> dst[i], int32 CUDA tensors [n]. Returns the cache."""
    lib = api._lib or load_library()
    pl = _plan(desc)
    dev = _pool(pl, cache)
    n = src.numel() if isinstance(src, torch.Tensor) else -1
    _on(src, "src", (max(n, 0),), torch.int32, dev)
    _on(dst, "dst", (max(n, 0),), torch.int32, dev)
    _raise_on(lib.ssba_cache_copy(pl.ref, cache._ref, src.data_ptr(), dst.data_ptr(), n, _stream_ptr(stream)))
    return cache
