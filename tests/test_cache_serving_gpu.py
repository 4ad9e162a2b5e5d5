"""The cache's calls together, as a server makes them: growing, forked, truncated and compacted sequences over several layers,
on other streams, in graphs, and with a wait that runs out."""
import ctypes
import math
import threading

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_15684_gb300 import api, build
from paper_2605_15684_gb300 import cache as pc
from test_cache_gpu import BF16, FP32, Batch, hold, ints, queries, shares

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    api.load_library()


@pytest.fixture(autouse=True)
def _status():
    torch.cuda.synchronize()
    api.get_status()
    yield
    torch.cuda.synchronize()


class Model:
    """What a PagedCache is to hold: every sequence's own K and V, in a reference pool of its own pages."""

    def __init__(self, kv, d, layers):
        self.kv, self.d, self.layers, self.seqs = kv, d, layers, {}

    def _pool(self, pages):
        p = ref.Pool.__new__(ref.Pool)
        shape = (pages, self.kv, 64, self.d)
        p.K, p.V = np.zeros(shape), np.zeros(shape)
        p.k_scale, p.v_scale, p.k_mean = np.zeros(shape[:2]), np.zeros(shape[:2]), np.zeros((pages, self.kv, self.d))
        return p

    def new(self, s):
        self.seqs[s] = [0, [self._pool(16) for _ in range(self.layers)]]

    def fork(self, a, b):
        n, pools = self.seqs[a]
        copies = []
        for p in pools:
            q = ref.Pool.__new__(ref.Pool)
            q.__dict__ = {k: v.copy() for k, v in p.__dict__.items()}
            copies.append(q)
        self.seqs[b] = [n, copies]

    def append(self, s, layer, k, v):
        n, pools = self.seqs[s]
        ref.append(pools[layer], k, v, np.arange(16)[None], [n], [0, k.shape[0]])

    def attend(self, s, layer, q, n_after, lists=None):
        return ref.attend(self.seqs[s][1][layer], q, np.arange(16)[None], [n_after], [0, q.shape[0]], self.d ** -0.5, lists)


@pytest.mark.parametrize("dtype,d,heads,kv", [(BF16, 128, 8, 2), (BF16, 64, 3, 3), (FP32, 64, 4, 1)])
def test_server(dtype, d, heads, kv):
    """Random steps of several sequences in two layers: prompts, single tokens, drafts, forks, rejected drafts, ends, and
    compaction; every output against the reference's own copy of the sequence."""
    layers, rng = 2, np.random.default_rng(5)
    g = torch.Generator().manual_seed(7)
    cache, model = pc.PagedCache(pc.CacheDesc(heads, kv, d, 40, dtype), layers), Model(kv, d, layers)
    live = []
    for turn in range(30):
        if len(live) < 3 or rng.random() < 0.15:
            s = cache.new()
            model.new(s)
            live.append(s)
        elif rng.random() < 0.25:
            a = live[rng.integers(len(live))]
            s = cache.fork(a)
            model.fork(a, s)
            live.append(s)
        if len(live) > 5:
            s = live.pop(rng.integers(len(live)))
            cache.free(s)
            del model.seqs[s]
        if rng.random() < 0.2:
            s = live[rng.integers(len(live))]
            n = int(rng.integers(model.seqs[s][0] + 1))
            cache.truncate(s, n)
            model.seqs[s][0] = n
        if turn % 7 == 6:
            cache.compact()
            assert cache.table.free_pages == 40 - (max((p for s in live for p in cache.table.pages_of(s)), default=-1) + 1)
        some = [s for s in live if rng.random() < 0.8 and model.seqs[s][0] < 500]
        counts = [int(rng.choice([1, 1, 1, 5, 70])) for _ in some]
        if not some:
            continue
        step = cache.step(some, counts)
        cu = shares(counts)
        for layer in range(layers):
            k, v = (torch.randn((cu[-1], kv, d), generator=g).to(dtype) for _ in range(2))
            q = (torch.randn((cu[-1], heads, d), generator=g) * 1.5).to(dtype)
            cache.append(step, layer, k.cuda(), v.cuda())
            O, lse = cache.attend(step, layer, q.cuda())
            keep = 3
            lists = pc.cache_select(cache.desc, cache.pools[layer], q.cuda(), step.table, step.lens, step.cu, keep)
            O2, lse2 = cache.attend(step, layer, q.cuda(), keep=keep)
            torch.cuda.synchronize()
            assert api.get_status() == api.SSBA_OK
            for i, s in enumerate(some):
                r = slice(cu[i], cu[i + 1])
                model.append(s, layer, k[r].double().numpy(), v[r].double().numpy())
                n = model.seqs[s][0] + counts[i]
                for got, gl, li in ((O, lse, None), (O2, lse2, lists[0][r].cpu().numpy())):
                    want, wl, A, S = model.attend(s, layer, q[r].double().numpy(), n, li)
                    bO, bl = ref.bounds(want, A, S, d, n, dtype == BF16)
                    hold(got[r], want, bO, (turn, s, "O"))
                    hold(gl[r], wl, bl, (turn, s, "lse"))
        for s, n in zip(some, counts):
            model.seqs[s][0] += n
            assert cache.length(s) == model.seqs[s][0]


def args(bt, n, heads, seed=1):
    cu = shares(n)
    return bt.desc(heads), bt.cache, queries(cu[-1], heads, bt.d, BF16, seed), bt.gpu_table(), ints(bt.lens), ints(cu)


def test_other_streams():
    """Calls on another stream while the current one is busy, with outputs and workspaces of the binding's."""
    bts = [Batch([3000, 500], 2, 128, 1), Batch([900, 70], 2, 128, 2)]
    calls = [args(bts[0], [1, 1], 8), args(bts[1], [40, 9], 8)]
    want = [(pc.cache_attend(*a), pc.cache_select(*a, 5)) for a in calls]
    torch.cuda.synchronize()
    busy = torch.randn(8192, 8192, device="cuda").bfloat16()
    for _ in range(3):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(10):
            busy @ busy
        got = []
        for a in calls:
            got.append((pc.cache_attend(*a, stream=s), pc.cache_select(*a, 5, stream=s)))
            junk = [torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        for x, y in zip(got, want):
            for p, q in zip(x, y):
                assert all(torch.equal(a, b) for a, b in zip(p, q))
    del junk


def test_results_do_not_depend_on_the_order_of_ctas():
    """Items that many CTAs share: the same bits every time, and beside other work."""
    for lens, n in (([9000, 31, 2500], [1, 1, 1]), ([2500, 700], [60, 33])):
        a = args(Batch(lens, 1, 128), n, 8)
        want = pc.cache_attend(*a)
        busy = torch.randn(2048, 2048, device="cuda").bfloat16()
        s = torch.cuda.Stream()
        for _ in range(20):
            with torch.cuda.stream(s):
                busy @ busy
            got = pc.cache_attend(*a)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.cuda.synchronize()


def test_two_graphs_side_by_side():
    """Two graphs of the same calls, captured before any other and replayed at once: neither's workspace is the other's, nor
    that of calls outside."""
    pc._ws.clear()
    a = args(Batch([5000, 2000], 1, 128), [1, 1], 8)
    b = args(Batch([1500, 600], 1, 64), [90, 20], 6, 2)
    graphs = []
    for x in (a, b, a):
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = [pc.cache_attend(*x) for _ in range(3)]
        graphs.append((s, g, out, x))
    want = {id(x): pc.cache_attend(*x) for x in (a, b)}
    torch.cuda.synchronize()
    for _ in range(5):
        for s, g, _, _ in graphs:
            with torch.cuda.stream(s):
                g.replay()
        outside = pc.cache_attend(*a)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        for _, _, out, x in graphs:
            for O, lse in out:
                assert torch.equal(O, want[id(x)][0]) and torch.equal(lse, want[id(x)][1])
        assert torch.equal(outside[0], want[id(a)][0])


def test_a_captured_step_with_new_lengths():
    """A decoding step in a graph: append, select and attend; lens, tokens and rows change between replays."""
    bt = Batch([0, 0, 0], 2, 128, pool_lens=[400, 200, 130])
    pool = bt.pool()
    lens = [70, 0, 129]
    k0 = torch.randn((sum(lens), 2, 128)).bfloat16()
    cu = shares(lens)
    pc.cache_append(bt.desc(8), bt.cache, k0.cuda(), k0.flip(0).contiguous().cuda(), bt.gpu_table(), ints([0, 0, 0]), ints(cu))
    ref.append(pool, k0.double().numpy(), k0.flip(0).double().numpy(), bt.table, [0, 0, 0], cu)
    T = 3
    k, v, q = (torch.zeros((T, h, 128), dtype=BF16, device="cuda") for h in (2, 2, 8))
    table, held, now, cud = bt.gpu_table(), ints([0, 0, 0]), ints([1, 1, 1]), ints([0, 1, 2, 3])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pc.cache_append(bt.desc(8), bt.cache, k, v, table, held, cud)
        idx, cnt = pc.cache_select(bt.desc(8), bt.cache, q, table, now, cud, 2)
        O, lse = pc.cache_attend(bt.desc(8), bt.cache, q, table, now, cud)
        O2, lse2 = pc.cache_attend(bt.desc(8), bt.cache, q, table, now, cud, idx, cnt)
    for turn in range(12):
        rows = shares([1, 1, 1] if turn % 3 else [1, 0, 1])  # a padded batch: the last row belongs to none
        n = [b - a for a, b in zip(rows, rows[1:])]
        gen = torch.Generator().manual_seed(turn)
        kn, vn, qn = (torch.randn((T, h, 128), generator=gen).bfloat16() for h in (2, 2, 8))
        k.copy_(kn), v.copy_(vn), q.copy_(qn)
        held.copy_(ints(lens)), now.copy_(ints([a + b for a, b in zip(lens, n)])), cud.copy_(ints(rows))
        g.replay()
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        ref.append(pool, kn.double().numpy(), vn.double().numpy(), bt.table, lens, rows)
        lens = [a + b for a, b in zip(lens, n)]
        e = rows[-1]
        for got, gl, li in ((O, lse, None), (O2, lse2, idx.cpu().numpy())):
            want, wl, A, S = ref.attend(pool, qn.double().numpy()[:e], bt.table, lens, rows, 128 ** -0.5, li)
            bO, bl = ref.bounds(want, A, S, 128, max(lens), True)
            hold(got[:e], want, bO, "O")
            hold(gl[:e], wl, bl, "lse")


@pytest.mark.parametrize("lens,n,d", [([3000, 100], [1, 1], 128), ([3000, 100], [1, 1], 64), ([900, 300], [60, 50], 128),
                                      ([900, 300], [60, 50], 64)])
def test_a_wait_that_runs_out(lens, n, d):
    """Copies that are announced and never come: the call ends with SSBA_ERR_TIMEOUT, the context and the binding's next
    call are well."""
    a = args(Batch(lens, 2, d), n, 8)
    want = pc.cache_attend(*a)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    ws = torch.zeros(pc.cache_attend_workspace_bytes(a[0]), dtype=torch.uint8, device="cuda")
    pc.test_cache_timeout(*a, torch.empty_like(want[0]), torch.empty_like(want[1]), ws)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_TIMEOUT
    got = pc.cache_attend(*a)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_timeout_is_not_hidden_by_a_later_check():
    """A wait that ran out, and behind it, before anyone has read the status, a call with a page outside the pool: what is
    read is the timeout, whose counters the binding has to forget."""
    for lens, n in (([3000, 100], [1, 1]), ([900, 300], [60, 50])):
        bt = Batch(lens, 2, 128)
        a = args(bt, n, 8)
        want = pc.cache_attend(*a)
        (kept,) = [w for (dev, st), w in pc._ws.items() if st == torch.cuda.current_stream().cuda_stream]
        pc.test_cache_timeout(*a, torch.empty_like(want[0]), torch.empty_like(want[1]), kept)
        table = bt.gpu_table()
        table[1, 0] = bt.pages
        other = torch.zeros(pc.cache_attend_workspace_bytes(a[0]), dtype=torch.uint8, device="cuda")
        pc.cache_attend(a[0], a[1], a[2], table, a[4], a[5], workspace=other)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_ERR_TIMEOUT
        got = pc.cache_attend(*a)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_workspace_is_left_as_it_was_found():
    """The counters are zero after a call, so that a caller's workspace serves call after call of any shape."""
    ws = torch.zeros(pc.cache_attend_workspace_bytes(Batch([64], 1, 64).desc(1)), dtype=torch.uint8, device="cuda")
    for lens, n, heads, kv, d in (([9000], [1], 8, 1, 128), ([2000, 900], [50, 60], 4, 1, 64), ([9000, 3], [2, 1], 8, 2, 64)):
        a = args(Batch(lens, kv, d), n, heads)
        want = pc.cache_attend(*a)
        got = pc.cache_attend(*a, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert not ws[:4096].any()


def test_scores_of_every_size():
    """Rows whose weights span many powers of two: one dominating key far from the others, and scores that fall and rise
    along the sequence, so that references are raised again and again."""
    for d, n in ((128, 1), (64, 1), (128, 40), (64, 40)):
        bt = Batch([900], 1, d)
        # keys grow along the sequence: scales of pages from 2^-12 to 2^-2
        for j in range(15):
            bt.cache.k_scale[bt.table[0][j]] = 2.0 ** (-12 + (j * 7) % 11)
            bt.cache.v_scale[bt.table[0][j]] = 2.0 ** (-9 + (j * 5) % 13)
        q = queries(n, 4, d, BF16, 3)
        O, lse = pc.cache_attend(bt.desc(4), bt.cache, q, bt.gpu_table(), ints([900]), ints([0, n]))
        torch.cuda.synchronize()
        want, wl, A, S = ref.attend(bt.pool(), q.double().cpu().numpy(), bt.table, [900], [0, n], d ** -0.5)
        bO, bl = ref.bounds(want, A, S, d, 900, True)
        hold(O, want, bO, (d, n, "O"))
        hold(lse, wl, bl, (d, n, "lse"))


@pytest.mark.parametrize("n", [1, 40])
def test_one_token_that_dominates_many_small_ones(n):
    """An attention sink: the first token's weight is 2^13 times any other's, and the others together are most of O."""
    d, L = 64, 20000
    bt = Batch([L], 1, d)
    K, V = bt.cache.K.view(torch.uint8), bt.cache.V.view(torch.uint8)
    K.fill_(0)
    V.fill_(0x38)  # 1.0
    bt.cache.k_scale.fill_(1.0)
    bt.cache.v_scale.fill_(1.0)
    p0 = bt.table[0][0]
    K[p0, :, 0] = 0x38
    V[p0, :, 0] = 0
    q = torch.full((n, 2, d), 13 * math.log(2) / d ** 0.5, device="cuda").bfloat16()
    O, lse = pc.cache_attend(bt.desc(2), bt.cache, q, bt.gpu_table(), ints([L]), ints([0, n]))
    torch.cuda.synchronize()
    want, wl, A, S = ref.attend(bt.pool(), q.double().cpu().numpy(), bt.table, [L], [0, n], d ** -0.5)
    bO, bl = ref.bounds(want, A, S, d, L, True)
    assert 0.6 < want.min() <= want.max() < 0.8
    hold(O, want, bO, "O")
    hold(lse, wl, bl, "lse")


def test_short_and_long_way_into_a_call():
    """Outputs given or not, a stream given or not: the same results; and what is out of order is named either way."""
    bt = Batch([700, 90], 2, 128)
    desc, cache, q, table, lens, cu = a = args(bt, [1, 1], 8)
    short = (*pc.cache_select(*a, 4), *pc.cache_attend(*a))
    s = torch.cuda.current_stream()
    long = (*pc.cache_select(*a, 4, stream=s), *pc.cache_attend(*a, stream=s))
    torch.cuda.synchronize()
    for x, y in zip(short, long):
        assert x.shape == y.shape and x.dtype == y.dtype and torch.equal(x, y)
    O, lse = pc.cache_attend(*a, short[0], short[1])
    O2, lse2 = pc.cache_attend(*a, short[0], short[1], stream=s)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    bad = [(dict(q=q.float()), "dtype"), (dict(q=q[:, :4].contiguous()), "shape"), (dict(q=q.cpu()), "CUDA tensor"),
           (dict(q=q.repeat(1, 1, 2)[:, :, ::2]), "contiguous"), (dict(table=table.long()), "dtype"), (dict(lens=lens[:1]), "shape"),
           (dict(cu=cu[:2]), "shape"), (dict(idx=short[0]), "together"), (dict(idx=short[0], cnt=short[1][:1]), "shape"),
           (dict(cache=pc.cache_alloc(pc.CacheDesc(8, 2, 128, 3))), "expected"), (dict(desc=pc.CacheDesc(8, 1, 128, 3)), "expected")]
    for kw, what in bad:
        call = dict(desc=desc, cache=cache, q=q, table=table, lens=lens, cu=cu, idx=None, cnt=None)
        call.update(kw)
        for more in (dict(), dict(stream=s)):
            with pytest.raises(api.SsbaError, match=what):
                pc.cache_attend(**call, **more)
    with pytest.raises(api.SsbaError, match="more than first"):
        pc.cache_select(*a, 1)
    with pytest.raises(api.SsbaError, match="workspace"):
        pc.cache_attend(*a, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(api.SsbaError, match="workspace"):
        pc.cache_attend(*a, workspace=None)
    with pytest.raises(AttributeError):
        cache.K = cache.V
    k = torch.zeros((2, 2, 128), dtype=BF16, device="cuda")
    for kw, what in ((dict(k=k.float(), v=k), "dtype"), (dict(k=k, v=k[:1]), "shape"), (dict(k=k[:, :1].contiguous(), v=k), "shape")):
        with pytest.raises(api.SsbaError, match=what):
            pc.cache_append(desc, cache, kw["k"], kw["v"], table, lens, cu)
    with pytest.raises(api.SsbaError, match="dtype"):
        pc.cache_copy(desc, cache, cu.long(), cu.long())
    # nothing to do
    none = ints([0])
    O, lse = pc.cache_attend(desc, cache, q[:0], table[:0], lens[:0], none)
    idx, cnt = pc.cache_select(desc, cache, q[:0], table[:0], lens[:0], none, 4)
    pc.cache_append(desc, cache, k[:0], k[:0], table[:0], lens[:0], none)
    assert O.shape == (0, 8, 128) and lse.shape == (0, 8) and idx.shape == (0, 2, 4) and cnt.shape == (0, 2)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK


def test_calls_let_other_threads_run():
    """The native calls hold Python's lock neither while they allocate nor while they launch: entry points that are asked
    for it (a stand-in returns 1 where its thread holds it, 0, which is SSBA_OK, where not) say so."""
    bt = Batch([700, 90], 2, 128)
    desc, cache, q, table, lens, cu = args(bt, [1, 1], 8)
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    assert ctypes.pythonapi.PyGILState_Check() == 1
    c, ext = desc.c(), pc._extension()
    call = ext.bind(held, held, held, held, ctypes.addressof(c), ctypes.addressof(cache._c), q.device.index, True)
    k = torch.zeros((2, 2, 128), dtype=BF16, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert ext.append(call, k, k, table, lens, cu) == 0
    assert ext.copy(call, lens, lens) == 0
    assert isinstance(ext.select(call, q, table, lens, cu, 4, 1), tuple)
    assert isinstance(ext.attend(call, q, table, lens, cu, None, None, ws), tuple)


def test_threads_with_streams_of_their_own():
    """Threads that serve sequences of their own side by side, each on its stream: what each would get alone."""
    def work(i, out):
        torch.cuda.set_device(0)
        with torch.cuda.stream(torch.cuda.Stream()):
            desc, cache, q, table, lens, cu = a = calls[i]
            for _ in range(25):
                O, lse = pc.cache_attend(*a)
                idx, cnt = pc.cache_select(*a, 4)
                O2, lse2 = pc.cache_attend(*a, idx, cnt)
            out[i] = (O, lse, idx, cnt, O2, lse2)
            torch.cuda.current_stream().synchronize()

    batches = [Batch([3000 - 500 * i, 90 + i], 2, 128 if i % 2 else 64, i) for i in range(4)]
    calls = [args(bt, [1, 1] if i < 2 else [50, 9], 8) for i, bt in enumerate(batches)]
    torch.cuda.synchronize()
    alone, together = {}, {}
    for i in range(4):
        work(i, alone)
    threads = [threading.Thread(target=work, args=(i, together)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    for i in range(4):
        assert all(torch.equal(x, y) for x, y in zip(alone[i], together[i]))


@pytest.mark.parametrize("B", [129, 1500])
def test_large_batches(B):
    """More sequences than a CTA has threads, and than one pass counts: append, select, attend."""
    lens = [(37 * b) % 200 + (b % 3 > 0) for b in range(B)]
    bt = Batch([0] * B, 1, 64, pool_lens=[n + 70 for n in lens], width=5)
    pool = bt.pool()
    g = torch.Generator().manual_seed(1)
    cu = shares(lens)
    k, v = (torch.randn((cu[-1], 1, 64), generator=g).bfloat16() for _ in range(2))
    zero = [0] * B
    pc.cache_append(bt.desc(2), bt.cache, k.cuda(), v.cuda(), bt.gpu_table(), ints(zero), ints(cu))
    n = [1 if b % 5 else 3 for b in range(B)]
    cu1 = shares(n)
    k1, v1 = (torch.randn((cu1[-1], 1, 64), generator=g).bfloat16() for _ in range(2))
    pc.cache_append(bt.desc(2), bt.cache, k1.cuda(), v1.cuda(), bt.gpu_table(), ints(lens), ints(cu1))
    torch.cuda.synchronize()
    ref.append(pool, k.double().numpy(), v.double().numpy(), bt.table, zero, cu)
    ref.append(pool, k1.double().numpy(), v1.double().numpy(), bt.table, lens, cu1)
    got = bt.pool()
    for name in ("K", "V", "k_scale", "v_scale", "k_mean"):
        assert np.array_equal(getattr(got, name), getattr(pool, name), equal_nan=True), name
    now = [a + b for a, b in zip(lens, n)]
    q = queries(cu1[-1], 2, 64, BF16, 4)
    idx, cnt = pc.cache_select(bt.desc(2), bt.cache, q, bt.gpu_table(), ints(now), ints(cu1), 2)
    for li in (None, idx):
        O, lse = pc.cache_attend(bt.desc(2), bt.cache, q, bt.gpu_table(), ints(now), ints(cu1), li, None if li is None else cnt)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        want, wl, A, S = ref.attend(pool, q.double().cpu().numpy(), bt.table, now, cu1, 0.125, None if li is None else li.cpu().numpy())
        bO, bl = ref.bounds(want, A, S, 64, max(now), True)
        hold(O, want, bO, "O")
        hold(lse, wl, bl, "lse")


def test_a_pool_past_32_bits():
    """Pages whose bytes lie behind 2^31 and 2^32 of K and V: appended, copied, selected and read."""
    kv, d, pages = 8, 128, 70000  # 4.6 GB a tensor
    desc = pc.CacheDesc(16, kv, d, pages)
    cache = pc.cache_alloc(desc)
    far = [pages - 1, 33000, 65600, 3, 40000]
    table = ints([far[:3]])
    k, v = (torch.randn((150, kv, d), device="cuda").bfloat16() for _ in range(2))
    pc.cache_append(desc, cache, k, v, table, ints([0]), ints([0, 150]))
    pc.cache_copy(desc, cache, ints([far[1]]), ints([far[4]]))
    table = ints([[far[0], far[4], far[2]]])
    small = Batch([0], kv, d, pool_lens=[150])
    sd = small.desc(16)
    pc.cache_append(sd, small.cache, k, v, small.gpu_table(), ints([0]), ints([0, 150]))
    for n in (1, 30):
        q = queries(n, 16, d, BF16)
        want = pc.cache_attend(sd, small.cache, q, small.gpu_table()[:, :3].contiguous(), ints([150]), ints([0, n]))
        got = pc.cache_attend(desc, cache, q, table, ints([150]), ints([0, n]))
        lists = pc.cache_select(desc, cache, q, table, ints([150]), ints([0, n]), 2)
        ref_l = pc.cache_select(sd, small.cache, q, small.gpu_table()[:, :3].contiguous(), ints([150]), ints([0, n]), 2)
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        for x, y in zip((*got, *lists), (*want, *ref_l)):
            assert torch.equal(x, y)
    qf = queries(2, 16, d, FP32)
    df = pc.CacheDesc(16, kv, d, pages, FP32)
    got = pc.cache_attend(df, cache, qf, table, ints([150]), ints([0, 2]))
    want = pc.cache_attend(small.desc(16, FP32), small.cache, qf, small.gpu_table()[:, :3].contiguous(), ints([150]), ints([0, 2]))
    assert torch.equal(got[0], want[0])
