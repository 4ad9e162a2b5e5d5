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
import importlib.util
import os
from dataclasses import dataclass

import torch

from . import api, build
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
    __slots__ = ("K", "V", "k_scale", "v_scale", "k_mean", "_shape", "_dev", "_ref", "_c", "_calls")

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
        put(self, "_calls", {})

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


_ext = None


def _extension():
    """The native short way into the calls (csrc/host/cache_call.cpp), made by build() beside the library."""
    global _ext
    with _lock:
        if _ext is None:
            path = build.call_file()
            if not os.path.exists(path):
                raise SsbaError(api.SSBA_ERR_CUDA, f"{path} is missing: run paper_2605_15684_gb300.build.build()")
            spec = importlib.util.spec_from_file_location("_cache_call", path)
            ext = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(ext)
            _ext = ext
    return _ext


def _call(pl: _Plan, cache: Cache):
    """What the native calls take for this descriptor and pool; None where the pool is not the descriptor's."""
    if cache.__class__ is not Cache or cache._shape != pl.shape:
        return None
    call = cache._calls.get(pl)
    if call is None:
        lib, ext = load_library(), _extension()
        fns = [ctypes.cast(getattr(lib, "ssba_cache_" + n), ctypes.c_void_p).value for n in ("append", "select", "attend", "copy")]
        call = ext.bind(*fns, ctypes.addressof(pl.c), ctypes.addressof(cache._c), cache._dev.index,
                        pl.dtype is torch.bfloat16)
        cache._calls[pl] = call
    return call


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
    pl = _plan(desc)
    if stream is None:
        call = _call(pl, cache)
        rc = _ext.append(call, k, v, table, lens, cu) if call is not None else None
        if rc == 0:
            return cache
        if rc is not None:
            _raise_on(rc)
    lib = load_library()
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
    pl = _plan(desc)
    if stream is None and idx is None and cnt is None:
        call = _call(pl, cache)
        out = _ext.select(call, q, table, lens, cu, keep, first) if call is not None else None
        if out.__class__ is tuple:
            return out
        if out is not None:
            _raise_on(out)
    lib = load_library()
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
api._timed_out.append(_ws.clear)  # counters that a timeout has left set
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
    pl = _plan(desc)
    if stream is None and O is None and lse is None and workspace.__class__ is str:
        call = _call(pl, cache)
        if call is not None and cache._dev.index == torch._C._cuda_getDevice():
            out = _ext.attend(call, q, table, lens, cu, idx, cnt, _default_workspace(pl, api._lib, cache._dev, None, None))
            if out.__class__ is tuple:
                return out
            if out is not None:
                _raise_on(out)
    lib = load_library()
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


def test_cache_timeout(desc: CacheDesc, cache: Cache, q, table, lens, cu, O, lse, workspace, budget_ns: int = 2_000_000,
                       stream=None) -> None:
    """ssba_test_cache_timeout: the attention's failure-detection test hook (include/ssba.h)."""
    lib = load_library()
    pl = _plan(desc)
    dev = _pool(pl, cache)
    T = _rows(q, "q", pl.heads, pl, dev)
    batch = _batch(table, lens, cu, dev)
    _on(O, "O", q.shape, pl.dtype, dev)
    _on(lse, "lse", (T, pl.heads), torch.float32, dev)
    wp, wn = api._ws_args(workspace)
    _raise_on(lib.ssba_test_cache_timeout(pl.ref, cache._ref, q.data_ptr(), T, *batch, O.data_ptr(), lse.data_ptr(), wp,
                                          wn, int(budget_ns), _stream_ptr(stream)))


def cache_copy(desc: CacheDesc, cache: Cache, src, dst, stream=None) -> Cache:
    """ssba_cache_copy: pages src[i] -> dst[i], int32 CUDA tensors [n]. Returns the cache."""
    pl = _plan(desc)
    if stream is None:
        call = _call(pl, cache)
        rc = _ext.copy(call, src, dst) if call is not None else None
        if rc == 0:
            return cache
        if rc is not None:
            _raise_on(rc)
    lib = load_library()
    dev = _pool(pl, cache)
    n = src.numel() if isinstance(src, torch.Tensor) else -1
    _on(src, "src", (max(n, 0),), torch.int32, dev)
    _on(dst, "dst", (max(n, 0),), torch.int32, dev)
    _raise_on(lib.ssba_cache_copy(pl.ref, cache._ref, src.data_ptr(), dst.data_ptr(), n, _stream_ptr(stream)))
    return cache


class PageTable:
    """Which pages hold which sequence: the host's bookkeeping of one pool, without any tensor. A page belongs to one
    sequence or is shared by the forks of one; a shared page is copied before one of them writes to it."""

    def __init__(self, pages: int):
        if pages <= 0:
            raise SsbaError(SSBA_ERR_INVALID, f"pages={pages} must be positive")
        self.pages = pages
        self._free = list(range(pages - 1, -1, -1))  # taken from the end: low pages first
        self._users = [0] * pages
        self._seqs: dict = {}  # id -> [pages, tokens]
        self._next = 0

    @property
    def free_pages(self) -> int:
        return len(self._free)

    @property
    def sequences(self):
        return list(self._seqs)

    def _seq(self, seq: int):
        if seq not in self._seqs:
            raise SsbaError(SSBA_ERR_INVALID, f"no sequence {seq}")
        return self._seqs[seq]

    def length(self, seq: int) -> int:
        """Tokens of a sequence."""
        return self._seq(seq)[1]

    def pages_of(self, seq: int):
        return list(self._seq(seq)[0])

    def new(self) -> int:
        """An empty sequence's id."""
        self._seqs[self._next] = [[], 0]
        self._next += 1
        return self._next - 1

    def fork(self, seq: int) -> int:
        """A sequence that begins with all of another's tokens, on the same pages."""
        pages, n = self._seq(seq)
        new = self.new()
        self._seqs[new] = [list(pages), n]
        for p in pages:
            self._users[p] += 1
        return new

    def _drop(self, pages) -> None:
        for p in pages:
            self._users[p] -= 1
            if self._users[p] == 0:
                self._free.append(p)

    def free(self, seq: int) -> None:
        """Ends a sequence; its pages that nobody else uses are free."""
        self._drop(self._seq(seq)[0])
        del self._seqs[seq]

    def truncate(self, seq: int, tokens: int) -> None:
        """Keeps the first tokens of a sequence (a rejected draft)."""
        s = self._seq(seq)
        if not 0 <= tokens <= s[1]:
            raise SsbaError(SSBA_ERR_INVALID, f"sequence {seq} has {s[1]} tokens, not {tokens}")
        keep = -(-tokens // PAGE)
        self._drop(s[0][keep:])
        s[0], s[1] = s[0][:keep], tokens

    def grow(self, seqs, counts):
        """Room for counts[i] more tokens of each sequence. Returns the copies (src, dst) that have to be made before they are
        written: of last pages that others use too. Changes nothing when pages do not suffice."""
        if len(set(seqs)) != len(seqs) or len(seqs) != len(counts) or any(n < 0 for n in counts):
            raise SsbaError(SSBA_ERR_INVALID, "sequences come once each, with a count >= 0")
        plan, need, left = [], 0, {}
        for seq, n in zip(seqs, counts):
            pages, held = self._seq(seq)
            more = -(-(held + n) // PAGE) - len(pages)
            shared = False
            if n > 0 and held % PAGE:  # (of the forks that write to one page here, the last one left keeps it)
                users = left.get(pages[-1], self._users[pages[-1]])
                shared = users > 1
                left[pages[-1]] = users - shared
            plan.append((more, shared))
            need += more + shared
        if need > len(self._free):
            raise SsbaError(SSBA_ERR_WORKSPACE, f"{need} pages are needed, {len(self._free)} are free")
        copies = []
        for seq, n, (more, shared) in zip(seqs, counts, plan):
            s = self._seqs[seq]
            if shared:
                p = self._take()
                copies.append((s[0][-1], p))
                self._users[s[0][-1]] -= 1
                s[0][-1] = p
            s[0].extend(self._take() for _ in range(more))
            s[1] += n
        return copies

    def _take(self) -> int:
        p = self._free.pop()
        self._users[p] = 1
        return p

    def compact(self):
        """Live pages to the front of the pool. Returns the moves (src, dst); no page is in both."""
        live = sum(u > 0 for u in self._users)
        to = [p for p in range(live) if self._users[p] == 0]
        moves = dict(zip((p for p in range(live, self.pages) if self._users[p] > 0), to))
        for s in self._seqs.values():
            s[0] = [moves.get(p, p) for p in s[0]]
        for a, b in moves.items():
            self._users[b], self._users[a] = self._users[a], 0
        self._free = list(range(self.pages - 1, live - 1, -1))
        return list(moves.items())


@dataclass
class CacheStep:
    """The new tokens of some sequences, as the calls of every layer take them: table [B, width], held [B] tokens before
    the step, lens [B] with it, cu [B + 1] rows; int32 on the device. It names pages: good until one of its sequences is
    freed, truncated or takes another step, or the pools are compacted."""
    table: torch.Tensor
    held: torch.Tensor
    lens: torch.Tensor
    cu: torch.Tensor
    rows: int


class PagedCache:
    """The K/V cache of a model's layers: a pool a layer, and one page table for all of them.

        cache = PagedCache(CacheDesc(heads, kv_heads, head_dim, pages), layers)
        a = cache.new()
        step = cache.step([a], [k.shape[0]])            # pages for the new tokens
        for layer in range(layers):
            cache.append(step, layer, k, v)
            O, lse = cache.attend(step, layer, q)       # keep=64: only the 64 pages selected for each query
        b = cache.fork(a)                               # shares a's pages

    All its calls belong on one stream: pages are reused in the order of that stream."""

    def __init__(self, desc: CacheDesc, layers: int = 1, device="cuda"):
        self.desc = desc
        self.table = PageTable(desc.pages)
        self.pools = [cache_alloc(desc, device) for _ in range(layers)]
        self.device = self.pools[0].K.device

    def new(self) -> int:
        return self.table.new()

    def fork(self, seq: int) -> int:
        return self.table.fork(seq)

    def free(self, seq: int) -> None:
        self.table.free(seq)

    def truncate(self, seq: int, tokens: int) -> None:
        self.table.truncate(seq, tokens)

    def length(self, seq: int) -> int:
        return self.table.length(seq)

    @property
    def free_pages(self) -> int:
        return self.table.free_pages

    def _ints(self, x) -> torch.Tensor:
        return torch.tensor(x, dtype=torch.int32).to(self.device, non_blocking=True)

    def _copy(self, pairs) -> None:
        if pairs:
            with torch.cuda.device(self.device):  # (the page table has them already: no refusal for the current device's sake)
                src, dst = (self._ints(x) for x in zip(*pairs))
                for pool in self.pools:
                    cache_copy(self.desc, pool, src, dst)

    def compact(self) -> int:
        """Moves the live pages to the front of the pools; returns how many moved."""
        moves = self.table.compact()
        self._copy(moves)
        return len(moves)

    def step(self, seqs, counts) -> CacheStep:
        """Makes room for counts[i] new tokens of sequence seqs[i], whose rows follow one another in k, v and q. Their
        K and V are to be appended, in every layer, before anything reads them."""
        seqs, counts = list(seqs), [int(n) for n in counts]
        self._copy(self.table.grow(seqs, counts))
        pages = [self.table.pages_of(s) for s in seqs]
        width = max(max(map(len, pages), default=0), 1)
        lens = [self.table.length(s) for s in seqs]
        cu = [0]
        for n in counts:
            cu.append(cu[-1] + n)
        table = torch.tensor([p + [-1] * (width - len(p)) for p in pages], dtype=torch.int32).reshape(len(seqs), width)
        return CacheStep(table.to(self.device, non_blocking=True), self._ints([a - n for a, n in zip(lens, counts)]),
                         self._ints(lens), self._ints(cu), cu[-1])

    def append(self, step: CacheStep, layer: int, k, v) -> None:
        """The step's K and V [rows, kv_heads, head_dim] into a layer's pool."""
        cache_append(self.desc, self.pools[layer], k, v, step.table, step.held, step.cu)

    def attend(self, step: CacheStep, layer: int, q, keep: int | None = None, first: int = 1):
        """Attention of the step's queries [rows, heads, head_dim] over a layer's pool; with keep, over the pages that
        cache_select picks for each of them. Returns (O, lse)."""
        lists = (None, None)
        if keep is not None:
            lists = cache_select(self.desc, self.pools[layer], q, step.table, step.lens, step.cu, keep, first)
        return cache_attend(self.desc, self.pools[layer], q, step.table, step.lens, step.cu, *lists)
