"""The paged 8-bit cache on the GPU against plain 64-bit loops (tests/cache_ref.py)."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2605_15684_gb300 import api, build
from paper_2605_15684_gb300 import cache as pc

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    api.load_library()
    yield
    torch.cuda.synchronize()


@pytest.fixture(autouse=True)
def _status():
    api.get_status()
    yield


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def shares(n):
    cu = [0]
    for m in n:
        cu.append(cu[-1] + m)
    return cu


class Batch:
    """Sequences of `lens` tokens in a pool of random values on a grid (see perf/operators.py for why), every
    byte, scale and mean that no sequence holds set to NaN."""

    def __init__(self, lens, kv, d, seed=0, spare=3, width=None, pool_lens=None):
        g = torch.Generator().manual_seed(seed)
        held = pool_lens or lens
        need = [-(-L // ref.PAGE) for L in held]
        self.width = width or max(max(need), 1) + 1
        pages = sum(need) + spare
        perm = torch.randperm(pages, generator=g).tolist()
        self.table = np.full((len(lens), self.width), -7, dtype=np.int64)
        nan = lambda *s: torch.full(s, math.nan)
        K, V = (torch.full((pages, kv, 64, d), 0x7F, dtype=torch.uint8).view(ref.E4M3) for _ in range(2))
        ks, vs, km = nan(pages, kv), nan(pages, kv), nan(pages, kv, d)
        at = 0
        for b, L in enumerate(held):
            for j in range(need[b]):
                p = perm[at]
                at += 1
                self.table[b][j] = p
                m = min(64, L - 64 * j)
                shared = (torch.randn((kv, 1, d), generator=g) * 4).round() / 8
                x = (torch.randn((kv, m, d), generator=g) * 8).round().clamp(-32, 32) / 8 + shared.clamp(-1.5, 1.5)
                K[p, :, :m] = (x * 64).to(ref.E4M3)
                V[p, :, :m] = (torch.randn((kv, m, d), generator=g) * 64).clamp(-440, 440).to(ref.E4M3)
                ks[p] = torch.exp2(torch.randint(-7, -4, (kv,), generator=g).float())
                vs[p] = torch.exp2(torch.randint(-7, -4, (kv,), generator=g).float())
                if m == 64:
                    km[p] = K[p].float().mean(1) * ks[p][:, None]
        self.pages, self.kv, self.d, self.lens = pages, kv, d, list(lens)
        self.cache = pc.Cache(*(t.cuda() for t in (K, V, ks, vs, km)))

    def desc(self, heads, dtype=BF16, **kw):
        return pc.CacheDesc(heads, self.kv, self.d, self.pages, dtype, **kw)

    def pool(self):
        return ref.Pool(self.cache.K, self.cache.V, self.cache.k_scale, self.cache.v_scale, self.cache.k_mean)

    def gpu_table(self):
        return ints(self.table)


def queries(T, heads, d, dtype, seed=1, std=1.5):
    g = torch.Generator().manual_seed(seed)
    return ((torch.randn((T, heads, d), generator=g) * 8 * std).round().clamp(-56, 56) / 8).to(dtype).cuda()


def hold(got, want, bound, what):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    off = np.abs(got - want)[fine] / np.broadcast_to(bound, want.shape)[fine]
    assert off.size == 0 or off.max() <= 1, (what, float(off.max()))


def check_attend(bt, n, heads, dtype=BF16, lists=None, q=None, T_more=0, scale=0.0, seed=1):
    cu = shares(n)
    T = cu[-1] + T_more
    q = queries(T, heads, bt.d, dtype, seed) if q is None else q
    desc = bt.desc(heads, dtype, softmax_scale=scale)
    O = torch.full((T, heads, bt.d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, heads), 7.0, device="cuda")
    idx, cnt = (None, None) if lists is None else lists
    pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), ints(bt.lens), ints(cu), idx, cnt, O=O, lse=lse)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    e = cu[-1]
    assert (O[e:] == 7).all() and (lse[e:] == 7).all()
    want = ref.attend(bt.pool(), q.double().cpu().numpy()[:e], bt.table, bt.lens, cu, scale or bt.d ** -0.5,
                      None if idx is None else idx.cpu().numpy())
    bO, bl = ref.bounds(want[0], want[2], want[3], bt.d, max(max(bt.lens), 1), dtype == BF16)
    hold(O[:e], want[0], bO, "O")
    hold(lse[:e], want[1], bl, "lse")
    return O, lse


# ----------------------------------------------------------------------------- attend
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1], [63], [64], [65], [127, 128, 129], [1, 700, 64, 0, 333]])
def test_attend_single_tokens(lens, d, dtype):
    check_attend(Batch(lens, 2, d), [1 if L else 0 for L in lens], 8, dtype)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 2), (7, 1), (12, 1), (16, 2), (24, 3), (40, 1), (72, 1)])
def test_attend_head_layouts(heads, kv):
    check_attend(Batch([200, 90, 1], kv, 128), [1, 1, 1], heads)
    check_attend(Batch([200, 90, 1], kv, 64), [3, 1, 1], heads)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_chunks(d, dtype):
    """Several new tokens a sequence: prompts without a past, chunks, none, and rows behind the last sequence."""
    check_attend(Batch([70, 200, 5, 130, 0, 300], 2, d), [70, 9, 5, 1, 0, 0], 6, dtype, T_more=3)


def test_attend_more_rows_than_tokens():
    """A sequence said to hold fewer tokens than it has rows: the first rows see nothing."""
    O, lse = check_attend(Batch([3, 0, 66], 2, 128), [5, 2, 68], 8)
    assert (O[:2] == 0).all() and (lse[:2] == -math.inf).all()


@pytest.mark.parametrize("d", [64, 128])
def test_attend_long(d):
    """Sequences that are split over many CTAs, beside short ones."""
    check_attend(Batch([9000, 31, 2500], 1, d), [1, 1, 1], 4)
    check_attend(Batch([5000], 2, d), [2], 16)


def test_attend_long_chunk():
    check_attend(Batch([1500, 640], 1, 128), [150, 33], 4)


def test_attend_many_short_sequences():
    lens = [(37 * b) % 150 + 1 for b in range(333)]
    check_attend(Batch(lens, 1, 64), [1] * 333, 2)


def test_attend_scale_and_peaks():
    """A softmax scale of its own, and scores so far apart that one key takes all the weight."""
    bt = Batch([300, 100], 2, 128)
    check_attend(bt, [1, 2], 8, scale=0.5)
    check_attend(bt, [1, 2], 8, FP32, scale=3.0)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_lists(dtype):
    bt = Batch([1000, 64, 130, 700], 2, 128)
    n = [2, 1, 1, 3]
    q = queries(7, 8, 128, dtype)
    lists = pc.cache_select(bt.desc(8, dtype), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints(shares(n)), 5)
    check_attend(bt, n, 8, dtype, lists, q)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("heads,kv,d", [(17, 1, 64), (40, 1, 128), (72, 2, 64), (12, 1, 128)])
def test_attend_lists_of_large_groups(heads, kv, d, dtype):
    """Groups that take several items of a few-row call, or several CTAs of an fp32 one, with lists."""
    bt = Batch([1000, 64, 130], kv, d, seed=71)
    n = [2, 1, 3]
    q = queries(6, heads, d, dtype, 72)
    lists = pc.cache_select(bt.desc(heads, dtype), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints(shares(n)), 4)
    check_attend(bt, n, heads, dtype, lists, q)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_lists_with_a_page_twice(dtype):
    """A page listed twice counts twice, the last one, which is not full, too."""
    bt = Batch([500, 290], 2, 128, seed=73)
    idx = ints([[[3, 7, 3, 0, 7], [1, -1, -1, -1, -1]], [[4, 4, 2, 2, 2], [0, 4, 0, 9, 9]]])
    check_attend(bt, [1, 1], 4, dtype, (idx, ints([[5, 1], [5, 3]])), seed=74)


@pytest.mark.parametrize("heads,kv", [(12, 1), (40, 1), (18, 2)])
def test_attend_fp32_large_groups(heads, kv):
    check_attend(Batch([200, 90, 1], kv, 128), [1, 1, 1], heads, FP32)
    check_attend(Batch([2500, 90, 1], kv, 64), [2, 1, 1], heads, FP32)


@pytest.mark.parametrize("heads,kv,d", [(130, 1, 64), (130, 1, 128), (256, 1, 64), (300, 1, 128), (600, 2, 64)])
def test_attend_groups_of_more_than_a_row_tile(heads, kv, d):
    """Groups past 128 rows of one token (two row tiles) and past 256 (several items), alone and joined from parts."""
    check_attend(Batch([200, 90, 1], kv, d, seed=75), [3, 1, 1], heads)
    check_attend(Batch([3000], kv, d, seed=76), [2], heads)


@pytest.mark.parametrize("n", [[0, 40, 0, 0, 1, 0], [0, 0, 0, 0, 0, 100]])
def test_attend_sequences_without_rows(n):
    """A padded batch: sequences that have tokens and no rows, in front, between and behind."""
    check_attend(Batch([300, 500, 0, 64, 70, 900], 2, 128, seed=77), n, 8, T_more=5, seed=78)


def test_attend_lists_of_nothing():
    """Empty lists, and lists of labels in any order."""
    bt = Batch([500, 500], 1, 64)
    idx, cnt = ints([[[6, 2, 0, -1]], [[-1, -1, -1, -1]]]), ints([[3], [0]])
    O, lse = check_attend(bt, [1, 1], 4, lists=(idx, cnt))
    assert (O[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_nan_behind_a_row(d, dtype):
    """NaN in tokens of the chunk that earlier rows do not see leave those rows alone, and reach the others."""
    bt = Batch([150], 2, d)
    page, slot = bt.table[0][146 // 64], 146 % 64
    bt.cache.V.view(torch.uint8)[page, 1, slot, 5] = 0x7F
    bt.cache.K.view(torch.uint8)[page, 0, slot + 2, 3] = 0xFF
    desc = bt.desc(4, dtype)
    q = queries(10, 4, d, dtype)
    O, lse = pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), ints([150]), ints([0, 10]))
    torch.cuda.synchronize()
    want, wl, A, S = ref.attend(bt.pool(), q.double().cpu().numpy(), bt.table, [150], [0, 10], d ** -0.5)
    # K/V head 1 (query heads 2, 3): rows 6.. see token 146 and its V; head 0: rows 8.. see the key of token 148
    assert np.isnan(want[6:, 2:, 5]).all() and np.isfinite(want[:, 2:, :5]).all() and np.isnan(want[8:, :2]).all()
    A, S = np.nan_to_num(A), np.nan_to_num(S)
    bO, bl = ref.bounds(np.nan_to_num(want), A, S, d, 150, dtype == BF16)
    hold(O, want, bO, "O")
    hold(lse, wl, bl, "lse")


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_pages_of_zeros_and_far_scales(d, dtype, n):
    """Pages whose K or V is all zero (scale 0), the first one too, beside V scales from 2^-60 to 2^30."""
    bt = Batch([700, 64, 300], 2, d, seed=31)
    c = bt.cache
    for b, zero_k, zero_v in ((0, (1, 4, 10), (0, 4, 7)), (1, (0,), (0,)), (2, (), (1, 4))):
        for j in zero_k:
            c.K.view(torch.uint8)[bt.table[b][j]] = 0
            c.k_scale[bt.table[b][j]] = 0
        for j in zero_v:
            c.V.view(torch.uint8)[bt.table[b][j]] = 0
            c.v_scale[bt.table[b][j]] = 0
    for j, e in ((1, -60), (2, 30), (5, -3), (9, 29)):
        c.v_scale[bt.table[0][j]] = 2.0 ** e
    check_attend(bt, [n, 1, min(n, 9)], 4, dtype, seed=32)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("zero,others", [((0,), -34), ((0, 5, 9), -44), ((0, 2), 28)])
def test_attend_pages_of_zero_values_beside_small_ones(zero, others, d, n):
    """Pages whose V is all zero, the first one among them, have a part in the weights' sum alone: the other pages' values,
    however small, keep their bits."""
    bt = Batch([700, 300], 2, d, seed=61)
    c = bt.cache
    for b in range(2):
        for j, p in enumerate(int(p) for p in bt.table[b] if p >= 0):
            c.v_scale[p] = 0.0 if j in zero else 2.0 ** others
            if j in zero:
                c.V.view(torch.uint8)[p] = 0
    check_attend(bt, [n, min(n, 33)], 4, seed=62)


# ----------------------------------------------------------------------------- select
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keep,first", [(1, 0), (2, 1), (5, 0), (9, 3), (30, 1)])
def test_select(keep, first, d, dtype):
    bt = Batch([1, 64, 65, 1500, 0, 640, 900], 2, d)
    n = [1, 1, 2, 1, 0, 3, 1]
    cu = shares(n)
    q = queries(cu[-1] + 2, 6, d, dtype)
    idx, cnt = (torch.full(s, 9, dtype=torch.int32, device="cuda") for s in ((cu[-1] + 2, 2, keep), (cu[-1] + 2, 2)))
    pc.cache_select(bt.desc(6, dtype), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints(cu), keep, first, idx, cnt)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    want = ref.select(bt.pool(), q.double().cpu().numpy(), bt.table, bt.lens, cu, keep, first)
    e = cu[-1]
    assert np.array_equal(idx[:e].cpu().numpy(), want[0][:e]) and np.array_equal(cnt[:e].cpu().numpy(), want[1][:e])
    assert (idx[e:] == 9).all() and (cnt[e:] == 9).all()


@pytest.mark.parametrize("pages", [257, 700, 2100])
def test_select_long(pages):
    """Long rows, with ties across the cut and pages of NaN."""
    bt = Batch([64 * pages - 5], 1, 64, spare=1)
    km = bt.cache.k_mean
    km[torch.from_numpy(bt.table[0][5:pages:9].copy()).cuda()] = 0.25
    km[torch.from_numpy(bt.table[0][7:pages:50].copy()).cuda()] = math.nan
    for keep, seed in ((16, 1), (200, 2), (pages - 1, 3), (pages - 20, 4)):
        q = queries(1, 4, 64, BF16, seed)
        idx, cnt = pc.cache_select(bt.desc(4), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints([0, 1]), keep)
        want = ref.select(bt.pool(), q.double().cpu().numpy(), bt.table, bt.lens, [0, 1], keep, 1)
        assert np.array_equal(idx.cpu().numpy(), want[0]) and np.array_equal(cnt.cpu().numpy(), want[1])


@pytest.mark.parametrize("keep,first", [(300, 128), (300, 129), (400, 399), (900, 517), (650, 0)])
def test_select_many_first_pages(keep, first):
    """More pages that are always kept than a CTA has threads."""
    bt = Batch([64 * 700, 64 * 401 + 1, 64 * 130], 1, 64, spare=1)
    q = queries(3, 2, 64, BF16, 5)
    idx, cnt = torch.full((3, 1, keep), -9, dtype=torch.int32, device="cuda"), torch.full((3, 1), -9, dtype=torch.int32, device="cuda")
    pc.cache_select(bt.desc(2), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints([0, 1, 2, 3]), keep, first, idx, cnt)
    want = ref.select(bt.pool(), q.double().cpu().numpy(), bt.table, bt.lens, [0, 1, 2, 3], keep, first)
    assert np.array_equal(idx.cpu().numpy(), want[0]) and np.array_equal(cnt.cpu().numpy(), want[1])


@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, FP32)])
def test_select_many_rows(d, dtype):
    """More rows than run at once."""
    lens = [(97 * b) % 700 + 1 for b in range(110)]
    bt = Batch(lens, 8, d, seed=8)
    q = queries(110, 16, d, dtype, 6)
    idx, cnt = pc.cache_select(bt.desc(16, dtype), bt.cache, q, bt.gpu_table(), ints(lens), ints(list(range(111))), 5, 1)
    want = ref.select(bt.pool(), q.double().cpu().numpy(), bt.table, lens, list(range(111)), 5, 1)
    assert np.array_equal(idx.cpu().numpy(), want[0]) and np.array_equal(cnt.cpu().numpy(), want[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keep", [3, 65, 700])
def test_select_few_high_scores_above_many_close_ones(keep, d):
    """Finite scores, a handful of which lie so far above that all others fall into the lowest steps between the extremes, where
    the cut then is: more of them than are ranked by counting. Sums of eighths and 64ths are exact in fp32."""
    pages, rows = 2200, 24
    bt = Batch([64 * pages - 7], 1, d, spare=1)
    g = torch.Generator().manual_seed(51)
    q = queries(rows, 4, d, BF16, 52)
    km = torch.randint(-2, 3, (pages, d), generator=g).float() / 64
    for i, j in enumerate((70, 700, 1500, 2100)):
        km[j] = q[i, i].float().cpu() * 256
    bt.cache.k_mean[torch.from_numpy(bt.table[0][:pages].copy()).cuda(), 0] = km.cuda()
    table = np.repeat(bt.table, rows, axis=0)
    lens, cu = [64 * pages - 7 - 64 * i for i in range(rows)], list(range(rows + 1))
    want = ref.select(bt.pool(), q.double().cpu().numpy(), table, lens, cu, keep, 1)
    for _ in range(20):
        idx, cnt = pc.cache_select(bt.desc(4), bt.cache, q, ints(table), ints(lens), ints(cu), keep)
        assert np.array_equal(idx.cpu().numpy(), want[0]) and np.array_equal(cnt.cpu().numpy(), want[1])
    assert api.get_status() == api.SSBA_OK


def test_select_all_equal():
    bt = Batch([64 * 40], 1, 128)
    bt.cache.k_mean.fill_(0.5)
    q = queries(1, 2, 128, BF16)
    idx, cnt = pc.cache_select(bt.desc(2), bt.cache, q, bt.gpu_table(), ints(bt.lens), ints([0, 1]), 7, 2)
    assert idx.tolist() == [[[0, 1, 2, 3, 4, 5, 39]]] and cnt.tolist() == [[7]]


# ----------------------------------------------------------------------------- append
def check_append(steps, kv, d, dtype, seed=0, std=1.0, width=None, edit=None):
    """Sequences grow by `steps` (lists of new tokens); after every step the pool equals the reference's."""
    B = len(steps[0])
    total = [sum(s[b] for s in steps) for b in range(B)]
    bt = Batch([0] * B, kv, d, seed, pool_lens=total, width=width)
    want = bt.pool()
    g = torch.Generator().manual_seed(seed + 99)
    lens = [0] * B
    for n in steps:
        cu = shares(n)
        k, v = (torch.randn((cu[-1] + 1, kv, d), generator=g) * std * 4.0 ** torch.randint(-3, 4, (cu[-1] + 1, kv, 1), generator=g)
                for _ in range(2))
        if edit:
            edit(k, v)
        k, v = k.to(dtype), v.to(dtype)
        before = [t.view(torch.uint8).clone() for t in (bt.cache.K, bt.cache.V)]
        pc.cache_append(bt.desc(kv, dtype), bt.cache, k.cuda(), v.cuda(), bt.gpu_table(), ints(lens), ints(cu))
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_OK
        ref.append(want, k.double().numpy(), v.double().numpy(), bt.table, lens, cu)
        got = bt.pool()
        for name in ("k_scale", "v_scale", "K", "V", "k_mean"):
            assert np.array_equal(getattr(got, name), getattr(want, name), equal_nan=True), name
        lens = [a + b for a, b in zip(lens, n)]
    return bt, lens


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_append(d, dtype):
    check_append([[1, 64, 0, 130, 63], [1, 1, 0, 1, 1], [62, 5, 3, 64, 1], [1, 0, 200, 127, 66]], 3, d, dtype)


def test_append_one_by_one():
    """Pages filled token by token, values growing and shrinking over twelve powers of two."""
    check_append([[1, 1]] * 70, 1, 64, BF16)


@pytest.mark.parametrize("dtype,std", [(BF16, 1e-30), (BF16, 1e30), (FP32, 1e-37), (FP32, 1e34)])
def test_append_ranges(dtype, std):
    check_append([[3, 64], [64, 1]], 1, 64, dtype, std=std)


def test_append_zeros_and_non_finite():
    def edit(k, v):
        k[0], v[0] = 0, 0
        if k.shape[0] > 3:
            k[1, 0, 3], v[1, 0, 4], k[2, 1, 0] = math.inf, -math.inf, math.nan
            v[3] = 0
    check_append([[1, 1], [70, 3], [1, 64]], 2, 64, BF16, edit=edit)


def test_append_again_over_the_same_tokens():
    """A step taken again from the same lens (a rejected draft) gives what it gave."""
    bt, lens = check_append([[70, 10]], 2, 128, BF16)
    k = torch.randn((6, 2, 128), device="cuda").bfloat16()
    args = (bt.desc(2), bt.cache, k, k, bt.gpu_table(), ints([64, 8]), ints([0, 4, 6]))
    pc.cache_append(*args)
    once = bt.pool()
    pc.cache_append(*args)
    again = bt.pool()
    for name in ("K", "V", "k_scale", "v_scale"):
        assert np.array_equal(getattr(again, name), getattr(once, name), equal_nan=True)


def test_append_values_of_every_exponent():
    """Rounding of values spread over e4m3's whole range under one scale, ties and subnormals among them."""
    x = torch.tensor([m / 16 * 2.0 ** e for e in range(-12, 9) for m in range(16, 32)] + [448.0] * 48)[:384]
    x = torch.cat([x, -x[:0]]).view(6, 1, 64)
    bt = Batch([0], 1, 64, pool_lens=[64])
    pool = bt.pool()
    pc.cache_append(bt.desc(1, FP32), bt.cache, x.cuda(), -x.cuda(), bt.gpu_table(), ints([0]), ints([0, 6]))
    torch.cuda.synchronize()
    ref.append(pool, x.double().numpy(), -x.double().numpy(), bt.table, [0], [0, 6])
    got = bt.pool()
    assert np.array_equal(got.K, pool.K, equal_nan=True) and np.array_equal(got.V, pool.V, equal_nan=True)


# ----------------------------------------------------------------------------- copy
@pytest.mark.parametrize("kv,d", [(1, 64), (3, 128), (24, 64)])
def test_copy(kv, d):
    bt = Batch([64 * 20 + 5], kv, d, spare=25)
    c = bt.cache
    perm = torch.randperm(bt.pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    src, dst = perm[:17].contiguous(), perm[17:34].contiguous()
    want = [t.view(torch.uint8).clone() for t in (c.K, c.V, c.k_scale, c.v_scale, c.k_mean)]
    for t in want:
        t[dst.long()] = t[src.long()]
    pc.cache_copy(bt.desc(kv), c, src, dst)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    for t, w in zip((c.K, c.V, c.k_scale, c.v_scale, c.k_mean), want):
        assert torch.equal(t.view(torch.uint8), w)
    pc.cache_copy(bt.desc(kv), c, src[:0], dst[:0])


# ----------------------------------------------------------------------------- what is out of range is left out
def test_bad_values_are_flagged_and_reach_nothing():
    """Pages outside the pool, lengths above the table, rows out of order, labels outside a row's pages: the
    status says so, and the rest of the batch is as it would be alone."""
    bt = Batch([200, 200], 1, 64)
    desc, lens, cu = bt.desc(2), ints([200, 200]), ints([0, 1, 2])
    q = queries(2, 2, 64, BF16)
    good, _ = pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), lens, cu)
    for bad in (-1, bt.pages, 2 ** 31 - 1, -2 ** 31):
        table = bt.gpu_table()
        table[0, 1] = bad
        O, lse = pc.cache_attend(desc, bt.cache, q, table, lens, cu)
        idx, cnt = pc.cache_select(desc, bt.cache, q, table, lens, cu, 3)
        assert torch.equal(O[1], good[1]) and torch.isfinite(O[0].float()).all()
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_ERR_CHECK
    for bad in (-5, 64 * bt.width + 1, 2 ** 31 - 1):
        O, _ = pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), ints([bad, 200]), cu)
        pc.cache_select(desc, bt.cache, q, bt.gpu_table(), ints([bad, 200]), cu, 3)
        assert torch.equal(O[1], good[1])
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_ERR_CHECK
    for bad in ([0, 5, 2], [-3, 1, 2], [0, 1, 9], [2, 1, 0]):
        pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), lens, ints(bad))
        pc.cache_select(desc, bt.cache, q, bt.gpu_table(), lens, ints(bad), 3)
        torch.cuda.synchronize()
    api.get_status()
    for bad in (-1, 4, 2 ** 31 - 1):
        idx = ints([[[0, bad, 2]], [[0, 1, 2]]])
        pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), lens, cu, idx, ints([[3], [3]]))
        torch.cuda.synchronize()
        assert api.get_status() == api.SSBA_ERR_CHECK
    pc.cache_attend(desc, bt.cache, q, bt.gpu_table(), lens, cu, ints([[[0, 1, 2]]] * 2), ints([[3], [4]]))
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_CHECK
    before = bt.pool()
    kk = torch.ones((2, 1, 64), dtype=BF16, device="cuda")
    table = bt.gpu_table()
    table[:, 3] = ints([bt.pages, -1])
    pc.cache_append(desc, bt.cache, kk, kk, table, lens, cu)  # token 200 goes to label 3
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_CHECK
    pc.cache_append(desc, bt.cache, kk, kk, bt.gpu_table(), ints([64 * bt.width] * 2), cu)  # no room
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_CHECK
    pc.cache_copy(desc, bt.cache, ints([0, -1]), ints([bt.pages, 1]))
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_CHECK
    after = bt.pool()
    for name in ("K", "V", "k_scale", "v_scale", "k_mean"):
        assert np.array_equal(getattr(after, name), getattr(before, name), equal_nan=True)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_queries_with_one_large_channel(d, n):
    """A channel of Q a thousand times the others', where K is zero: the others make the scores. 1000 is held
    as 250 * 4 in steps of 2^-9, so a row's small values are off by 2^-10 * 4 at most, which a score has d times over,
    times |k|; a weight is off by twice that, an output by A times that."""
    bt = Batch([900, 130], 2, d, seed=41)
    K = bt.cache.K.view(torch.uint8)
    K[..., 3] = 0
    g = torch.Generator().manual_seed(42)
    T = n + 1
    q = torch.randn((T, 8, d), generator=g)
    q[:, :, 3] = 1000 * torch.sign(q[:, :, 3])
    q = q.bfloat16().cuda()
    O, lse = pc.cache_attend(bt.desc(8), bt.cache, q, bt.gpu_table(), ints([900, 130]), ints([0, n, T]))
    torch.cuda.synchronize()
    want, wl, A, S = ref.attend(bt.pool(), q.double().cpu().numpy(), bt.table, [900, 130], [0, n, T], d ** -0.5)
    bO, bl = ref.bounds(want, A, S, d, 900, True)
    k = torch.nan_to_num(bt.cache.K.float() * bt.cache.k_scale[:, :, None, None]).abs().sum(-1).max().item()
    off = d ** -0.5 * k * 2.0 ** -10 * 4
    hold(O, want, bO + 2 * off * A, "O")
    hold(lse, wl, bl + off, "lse")


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_queries_hold_small_values_beside_a_large_one(d, n):
    """One channel of Q far above the others, where K is zero, for few rows and for many. The others are 4 (2^-5 + 2^-10),
    and 1000 is held as 250 * 4: what a value's first part leaves is 2^-10, the same in every channel, and keys have the
    queries' signs, so that nothing cancels. The two parts are off by 2^-14 * 4 at most, which a score has d times over,
    times |k|; a weight is off by twice that, an output by A times that."""
    bt = Batch([900, 130], 2, d, seed=41)
    c, T = bt.cache, n + 1
    g = torch.Generator().manual_seed(43)
    sign = torch.randint(0, 2, (d,), generator=g) * 2.0 - 1
    key = sign[None] * (32 + 4 * torch.randint(0, 8, (64, 1), generator=g).float())  # whole steps of e4m3
    key[:, 3] = 0
    c.K.view(torch.uint8)[:] = key.to(ref.E4M3).view(torch.uint8).cuda()
    c.k_scale.fill_(2.0 ** -4)
    q = (sign * 4 * (2.0 ** -5 + 2.0 ** -10)).repeat(T, 8, 1)
    q[:, :, 3] = 1000
    q = q.bfloat16().cuda()
    assert (q[:, :, 4].abs() == 4 * (2.0 ** -5 + 2.0 ** -10)).all()
    O, lse = pc.cache_attend(bt.desc(8), c, q, bt.gpu_table(), ints([900, 130]), ints([0, n, T]))
    torch.cuda.synchronize()
    want, wl, A, S = ref.attend(bt.pool(), q.double().cpu().numpy(), bt.table, [900, 130], [0, n, T], d ** -0.5)
    bO, bl = ref.bounds(want, A, S, d, 900, True)
    off = d ** -0.5 * d * 60 * 2.0 ** -4 * 2.0 ** -14 * 4
    hold(O, want, bO + 2 * off * A, "O")
    hold(lse, wl, bl + off, "lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,n,heads,kv", [([9000], [9], 8, 2), ([9000], [70], 8, 2), ([6000, 130, 2500], [300, 130, 77], 6, 3)])
def test_attend_rows_joined_from_parts(lens, n, heads, kv, d):
    # few rows of many parts and many rows of few: each item is shared out over several CTAs
    bt = Batch(lens, kv, d, seed=21)
    check_attend(bt, n, heads, seed=22)
    # which CTA joins an item depends on who is last; the result does not
    q, cu = queries(sum(n), heads, d, BF16, 23), ints(shares(n))
    first = pc.cache_attend(bt.desc(heads), bt.cache, q, bt.gpu_table(), ints(lens), cu)
    for _ in range(30):
        again = pc.cache_attend(bt.desc(heads), bt.cache, q, bt.gpu_table(), ints(lens), cu)
        for a, b in zip(first, again):
            assert torch.equal(a.view(torch.int16 if a.dtype == BF16 else torch.int32), b.view(torch.int16 if b.dtype == BF16 else torch.int32))
