"""Host-side checks of the paged cache's entry points (no compute call is made) and of the reference that
the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_15684_gb300 import api, build
from paper_2605_15684_gb300 import cache as pc

FAKE = 0x100000  # a 128-byte aligned, never dereferenced address


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load_library()


def desc(**kw):
    base = dict(heads=8, kv_heads=2, head_dim=128, pages=10, dtype=api.SSBA_BF16, softmax_scale=0.0)
    base.update(kw)
    return ctypes.byref(api._CacheDesc(**base))


def pool(**kw):
    base = dict(K=FAKE, V=FAKE, k_scale=FAKE, v_scale=FAKE, k_mean=FAKE)
    base.update(kw)
    return ctypes.byref(api._Cache(**base))


BATCH = (FAKE, 4, FAKE, FAKE, 2)  # table, width, lens, cu, B


def calls(lib, d, c, T=3, batch=BATCH):
    return (lib.ssba_cache_append(d, c, FAKE, FAKE, T, *batch, None),
            lib.ssba_cache_select(d, c, FAKE, T, *batch, 4, 1, FAKE, FAKE, None),
            lib.ssba_cache_attend(d, c, FAKE, T, *batch, None, None, 0, FAKE, FAKE, FAKE, 0, None))


@pytest.mark.parametrize("bad,code", [
    (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(heads=7), 1), (dict(pages=0), 1), (dict(dtype=5), 1),
    (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1),
    (dict(head_dim=0), 1), (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(heads=32768, kv_heads=8), 2),
    (dict(pages=2 ** 30, kv_heads=8), 2)])
def test_descriptors(lib, bad, code):
    assert set(calls(lib, desc(**bad), pool())) == {code}
    assert lib.ssba_cache_copy(desc(**bad), pool(), FAKE, FAKE, 1, None) == code
    assert lib.ssba_cache_attend_workspace_bytes(desc(**bad)) == 0
    assert lib.ssba_last_error()


@pytest.mark.parametrize("bad", [dict(K=None), dict(V=None), dict(k_scale=None), dict(v_scale=None), dict(k_mean=None),
                                 dict(K=FAKE + 16), dict(V=FAKE + 64), dict(k_scale=FAKE + 2), dict(k_mean=FAKE + 8)])
def test_pools(lib, bad):
    assert set(calls(lib, desc(), pool(**bad))) == {api.SSBA_ERR_INVALID}
    assert lib.ssba_cache_copy(desc(), pool(**bad), FAKE, FAKE, 1, None) == api.SSBA_ERR_INVALID
    assert set(calls(lib, desc(), None)) == {api.SSBA_ERR_INVALID}
    assert set(calls(lib, None, pool())) == {api.SSBA_ERR_INVALID}


@pytest.mark.parametrize("T,batch,code", [
    (-1, BATCH, 1), (3, (FAKE, 0, FAKE, FAKE, 2), 1), (3, (FAKE, 4, FAKE, FAKE, -1), 1), (3, (None, 4, FAKE, FAKE, 2), 1),
    (3, (FAKE, 4, None, FAKE, 2), 1), (3, (FAKE, 4, FAKE, None, 2), 1), (3, (FAKE + 2, 4, FAKE, FAKE, 2), 1),
    (2 ** 24 + 1, BATCH, 2), (3, (FAKE, 2 ** 25, FAKE, FAKE, 2), 2), (3, (FAKE, 4, FAKE, FAKE, 2 ** 24 + 1), 2)])
def test_batches(lib, T, batch, code):
    assert set(calls(lib, desc(), pool(), T, batch)) == {code}


def test_no_work_succeeds_without_a_device(lib):
    assert set(calls(lib, desc(), pool(), 0)) == {api.SSBA_OK}
    assert set(calls(lib, desc(), pool(), 3, (None, 4, None, None, 0))) == {api.SSBA_OK}
    assert lib.ssba_cache_copy(desc(), pool(), None, None, 0, None) == api.SSBA_OK


def test_outputs_lists_and_workspaces(lib):
    d, c = desc(), pool()
    sel = lambda q=FAKE, keep=4, first=1, idx=FAKE, cnt=FAKE, batch=BATCH: lib.ssba_cache_select(
        d, c, q, 3, *batch, keep, first, idx, cnt, None)
    for kw in (dict(q=None), dict(q=FAKE + 8), dict(keep=0, first=0), dict(keep=2, first=2), dict(first=-1), dict(idx=None),
               dict(cnt=None), dict(idx=FAKE + 1), dict(keep=32769)):
        assert sel(**kw) == api.SSBA_ERR_INVALID, kw
    assert sel(batch=(FAKE, 32769, FAKE, FAKE, 2)) == api.SSBA_ERR_UNSUPPORTED
    need = lib.ssba_cache_attend_workspace_bytes(d)
    assert need > 0
    att = lambda q=FAKE, idx=None, cnt=None, keep=0, O=FAKE, lse=FAKE, ws=FAKE, n=need: lib.ssba_cache_attend(
        d, c, q, 3, *BATCH, idx, cnt, keep, O, lse, ws, n, None)
    for kw in (dict(q=None), dict(O=None), dict(lse=None), dict(O=FAKE + 8), dict(idx=FAKE, keep=4), dict(cnt=FAKE, keep=4),
               dict(idx=FAKE, cnt=FAKE, keep=0), dict(idx=FAKE + 2, cnt=FAKE, keep=4)):
        assert att(**kw) == api.SSBA_ERR_INVALID, kw
    for kw in (dict(ws=None), dict(n=need - 1), dict(ws=FAKE + 8)):
        assert att(**kw) == api.SSBA_ERR_WORKSPACE, kw
    assert lib.ssba_cache_append(d, c, None, FAKE, 3, *BATCH, None) == api.SSBA_ERR_INVALID
    assert lib.ssba_cache_append(d, c, FAKE, FAKE + 4, 3, *BATCH, None) == api.SSBA_ERR_INVALID
    assert lib.ssba_cache_copy(d, c, None, FAKE, 1, None) == api.SSBA_ERR_INVALID
    assert lib.ssba_cache_copy(d, c, FAKE, FAKE, -1, None) == api.SSBA_ERR_INVALID


@pytest.mark.parametrize("dtype", [api.SSBA_BF16, api.SSBA_FP32])
def test_the_output_has_to_be_aligned_to_what_a_thread_writes_at_once(lib, dtype):
    d = desc(dtype=dtype)
    need = lib.ssba_cache_attend_workspace_bytes(d)
    for off in (4, 8, 16):
        assert lib.ssba_cache_attend(d, pool(), FAKE, 3, *BATCH, None, None, 0, FAKE + off, FAKE, FAKE, need,
                                     None) == api.SSBA_ERR_INVALID
        assert b"O 32-byte aligned" in lib.ssba_last_error()


def test_binding_refuses_before_it_calls(lib):
    d = pc.CacheDesc(8, 2, 128, 4)
    q, t = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(api.SsbaError, match="CUDA tensor"):
        pc.cache_alloc(d, "cpu")
    with pytest.raises(api.SsbaError, match="must be a Cache"):
        pc.cache_attend(d, None, q, t, t[0, :1], t[0, :2])
    with pytest.raises(api.SsbaError, match="dtype"):
        pc.cache_alloc(pc.CacheDesc(8, 2, 128, 4, torch.float16), "cpu")
    with pytest.raises(api.SsbaError, match="2\\^31"):
        pc.cache_alloc(pc.CacheDesc(2 ** 32 + 8, 2, 128, 4), "cpu")


# ----------------------------------------------------------------------------- the reference itself
def test_reference_bytes_and_rounding():
    """The table of values and the rounding equal torch's own e4m3."""
    b = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(ref.VALUES, b.view(ref.E4M3).double().numpy(), equal_nan=True)
    x = torch.cat([torch.randn(20000) * s for s in (100, 1, 0.01, 0.001)]).clamp(-448, 448)
    x = torch.cat([x, torch.arange(-448, 449) / 1.0, torch.arange(-1000, 1000) * 2.0 ** -11])
    assert np.array_equal(ref.round_e4m3(x.double().numpy()), x.to(ref.E4M3).double().numpy())


@pytest.mark.parametrize("a,s", [(0.0, 0.0), (448.0, 1.0), (448.001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (3.5, 2.0 ** -7),
                                 (3.6, 2.0 ** -6), (1e-45, 2.0 ** -126), (3e38, 2.0 ** 120)])
def test_reference_scale(a, s):
    assert ref.scale_for(a) == s


def test_reference_attention_is_a_softmax():
    """Against a dense softmax over contiguous values."""
    g = np.random.default_rng(0)
    p = ref.Pool.__new__(ref.Pool)
    p.K, p.V = g.normal(size=(3, 1, 64, 8)), g.normal(size=(3, 1, 64, 8))
    p.k_scale, p.v_scale, p.k_mean = np.full((3, 1), 0.5), np.full((3, 1), 2.0), None
    q = g.normal(size=(2, 2, 8))
    table = np.array([[2, 0]])
    O, lse, A, S = ref.attend(p, q, table, [100], [0, 2], 0.3)
    K = np.concatenate([p.K[2, 0], p.K[0, 0]]) * 0.5
    V = np.concatenate([p.V[2, 0], p.V[0, 0]]) * 2
    for i, L in ((0, 99), (1, 100)):
        a = 0.3 * q[i] @ K[:L].T
        w = np.exp(a) / np.exp(a).sum(1, keepdims=True)
        assert np.allclose(O[i], w @ V[:L], atol=1e-13) and np.allclose(lse[i], np.log(np.exp(a).sum(1)), atol=1e-13)


# ----------------------------------------------------------------------------- the host's page table
def check_table(t):
    """Every page is free or used by as many sequences as hold it."""
    users = [0] * t.pages
    for s in t.sequences:
        pages = t.pages_of(s)
        assert len(pages) == -(-t.length(s) // 64) and len(set(pages)) == len(pages)
        for p in pages:
            users[p] += 1
    assert users == t._users
    assert sorted(t._free) == [p for p in range(t.pages) if users[p] == 0]


def test_page_table_against_the_tokens_it_stands_for():
    """Random growing, forking, truncating, freeing and compacting: following the copies, every sequence reads its own tokens."""
    import random
    r = random.Random(3)
    for _ in range(30):
        t = pc.PageTable(r.randint(3, 40))
        mem = [[None] * 64 for _ in range(t.pages)]
        own, stamp = {}, 0
        for _ in range(120):
            what = r.random()
            if what < 0.15 or not own:
                own[t.new()] = []
            elif what < 0.3:
                s = r.choice(list(own))
                own[t.fork(s)] = list(own[s])
            elif what < 0.4:
                s = r.choice(list(own))
                t.free(s)
                del own[s]
            elif what < 0.5:
                s = r.choice(list(own))
                n = r.randint(0, len(own[s]))
                t.truncate(s, n)
                own[s] = own[s][:n]
            elif what < 0.55:
                moves = t.compact()
                assert not {a for a, _ in moves} & {b for _, b in moves}
                for a, b in moves:
                    mem[b] = list(mem[a])
                    mem[a] = [None] * 64
                assert t._free == list(range(t.pages - 1, t.pages - 1 - len(t._free), -1))
            else:
                some = [s for s in own if r.random() < 0.6]
                counts = [r.choice([0, 1, 1, 3, 64, 100]) for _ in some]
                before = (t.free_pages, {s: t.pages_of(s) for s in own})
                try:
                    copies = t.grow(some, counts)
                except api.SsbaError as e:
                    assert "free" in str(e)
                    assert before == (t.free_pages, {s: t.pages_of(s) for s in own})
                    continue
                for a, b in copies:
                    mem[b] = list(mem[a])
                for s, n in zip(some, counts):
                    for _ in range(n):
                        stamp += 1
                        at = len(own[s])
                        mem[t.pages_of(s)[at // 64]][at % 64] = stamp
                        own[s].append(stamp)
            check_table(t)
            for s, tokens in own.items():
                pages = t.pages_of(s)
                assert [mem[pages[i // 64]][i % 64] for i in range(len(tokens))] == tokens


def test_page_table_refusals():
    t = pc.PageTable(2)
    a, b = t.new(), t.new()
    for bad in (lambda: t.grow([a, a], [1, 1]), lambda: t.grow([a], [1, 2]), lambda: t.grow([a], [-1]), lambda: t.grow([9], [1]),
                lambda: t.grow([a, b], [64, 65]), lambda: t.truncate(a, 1), lambda: t.free(7), lambda: t.fork(7),
                lambda: pc.PageTable(0)):
        with pytest.raises(api.SsbaError):
            bad()
    check_table(t)
    assert t.grow([a, b], [64, 64]) == [] and t.free_pages == 0
    # two forks of one half-filled page: one copies, the other keeps it
    t = pc.PageTable(2)
    a = t.new()
    t.grow([a], [10])
    b = t.fork(a)
    assert len(t.grow([a, b], [1, 1])) == 1
    check_table(t)


def test_timeout_hook_validation(lib):
    need = lib.ssba_cache_attend_workspace_bytes(desc())
    call = lambda d, q=FAKE, ws=FAKE, n=need: lib.ssba_test_cache_timeout(d, pool(), q, 3, *BATCH, FAKE, FAKE, ws, n, 0, None)
    assert call(desc(dtype=api.SSBA_FP32)) == api.SSBA_ERR_UNSUPPORTED
    assert call(desc(), q=None) == api.SSBA_ERR_INVALID
    assert call(desc(), n=need - 1) == api.SSBA_ERR_WORKSPACE


def test_native_calls_leave_what_is_not_in_order_to_the_long_way(lib):
    """The extension loads without a GPU, and gives None for tensors that are not the call's; its errors are Python's."""
    ext = pc._extension()
    d = pc.CacheDesc(8, 2, 128, 10)
    pool_c = api._Cache(FAKE, FAKE, FAKE, FAKE, FAKE)
    call = ext.bind(FAKE, FAKE, FAKE, FAKE, ctypes.addressof(pc._plan(d).c), ctypes.addressof(pool_c), 0, True)
    q, t = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    if not torch.cuda.is_available():
        # (which device is current needs a driver: without one every call is left to the long way)
        assert ext.append(call, q, q, t, t, t) is None
        assert ext.select(call, q, t, t, t, 4, 1) is None
        assert ext.attend(call, q, t, t, t, None, None, t) is None
        assert ext.copy(call, t, t) is None
    assert ext.select(call, q, t, t, t, "x", 1) is None
    with pytest.raises(TypeError):
        ext.attend(call, q)
    with pytest.raises(ValueError):
        ext.append(None, q, q, t, t, t)


def test_copies_of_a_step_are_made_on_the_caches_device(monkeypatch):
    """The page table says that a step's pages were copied before they are: so that is done wherever the caller's current
    device is (calls on a pool refuse any but its own)."""
    current, made = ["another"], []

    class On:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.was, current[0] = current[0], self.dev

        def __exit__(self, *_):
            current[0] = self.was

    def copy(d, pool, src, dst, stream=None):
        if current[0] != cache.device:
            raise api.SsbaError(api.SSBA_ERR_INVALID, "the current device is another")
        made.append((pool, src.tolist(), dst.tolist()))

    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(pc, "cache_copy", copy)
    cache = object.__new__(pc.PagedCache)
    cache.desc, cache.table, cache.pools, cache.device = None, pc.PageTable(6), ["a", "b"], torch.device("cpu")
    a = cache.new()
    cache.step([a], [70])
    b = cache.fork(a)
    cache.step([b], [3])
    assert made == [("a", [1], [2]), ("b", [1], [2])] and cache.length(b) == 73
    cache.free(a)
    assert cache.compact() == 1 and made[2:] == [("a", [2], [1]), ("b", [2], [1])]
    assert current == ["another"]
