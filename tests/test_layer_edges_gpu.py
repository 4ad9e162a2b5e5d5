"""GPU tests of a layer's operators at their edges: values and layouts that are allowed and seldom met."""
import threading

import pytest
import torch

import paper_2605_15684_gb300 as gb
from paper_2605_15684_gb300 import api, build
from tests import layer_ref as ref
from tests.layer_ref import near

pytestmark = pytest.mark.gpu
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    api.load_library()
    yield
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK


def rng(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda") * std


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D,axes", [(64, (16,)), (96, (7, 11, 5)), (80, (12, 4, 4, 8)), (6, (2,)), (256, (100, 1)), (66, (32,))])
def test_rope_copies_the_dimensions_behind_its_pairs(D, axes, layout, dt):
    """Any bits there (infinities, NaN, -0 among them) come out as they went in and reach nothing else."""
    randn, tail = rng(D), 2 * sum(axes)
    g = torch.Generator(device="cuda").manual_seed(D)
    x = randn(2, 9, 7, D).to(dt)
    pos = torch.randint(-50, 2000, (9, len(axes)), generator=g, device="cuda", dtype=torch.int32)
    want = gb.rope_axes(x, pos, axes, layout=layout)
    if dt == BF:
        any_bits = torch.randint(-2 ** 15, 2 ** 15, (2, 9, 7, D - tail), generator=g, device="cuda").to(torch.int16)
    else:
        any_bits = torch.randint(-2 ** 31, 2 ** 31, (2, 9, 7, D - tail), generator=g, device="cuda").to(torch.int32)
    rest = any_bits.view(dt)
    rest[0, ..., 0], rest[0, ..., -1], rest[1, 0], rest[1, 1], rest[1, 2, 0] = float("inf"), float("-inf"), -0.0, float("nan"), float("inf")
    x[..., tail:] = rest
    for out in (None, x.clone(), torch.empty(2, 7, 9, D, device="cuda", dtype=dt).transpose(1, 2)):
        src = x if out is None or out.stride() != x.stride() else out
        y = gb.rope_axes(src, pos, axes, layout=layout, out=out)
        assert torch.equal(bits(y[..., tail:]), bits(rest))
        assert torch.equal(y[..., :tail], want[..., :tail])


def least_scale(y):
    """The least power of two (2^-126 at least) under which no finite value of y's rows (fp32) passes 448; 1 where all are 0."""
    a = torch.where(y.isfinite(), y, 0.0).abs().amax(1)
    m, e = torch.frexp(a)
    e = torch.where(a == 0, 0, (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126))
    return ((e.long() + 1023) << 52).view(torch.float64)


@pytest.mark.parametrize("D", [64, 256, 576, 784, 1600, 3136, 4096, 12544, 16384])
@pytest.mark.parametrize("dt", [BF, F32])
def test_e4m3_scale_at_its_border(D, dt):
    """One value a row and eps 0: y is sqrt(D) w whatever the value. With w = 7 / sqrt(D) it is 448 / 64 and the scale 2^-6; next to
    it above, twice that."""
    root = round(D ** 0.5)
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.zeros(256, D, device="cuda", dtype=dt)
    at = torch.randint(0, D, (256,), generator=g, device="cuda")
    x[torch.arange(256, device="cuda"), at] = (torch.randn(256, generator=g, device="cuda") * 4).to(dt)
    x[0, at[0]] = 1.2109375
    exact = root & (root - 1) == 0  # 7 / root is an fp32 number
    w7 = torch.full((D,), 7.0 / root if exact else 1.0, device="cuda")
    for w in (w7, torch.nextafter(w7, 2 * w7), torch.nextafter(w7, 0 * w7)):
        q, scale = gb.rms_norm(x, w, eps=0.0, e4m3=True)[:2]
        y = (ref.norm(x, w, 0.0)[0]).float()
        want = least_scale(y)
        assert torch.equal(scale.double(), want), (scale.double() / want).unique()
        assert torch.equal(q.float(), (y.double() / want[:, None]).float().to(E4M3).float())


@pytest.mark.parametrize("D", [64, 1536, 4096, 16384])
@pytest.mark.parametrize("dt", [BF, F32])
def test_e4m3_scale_of_odd_rows(D, dt):
    """Rows of zeros, of values that no e4m3 can follow, weights that underflow before rstd brings them back, NaN and infinities."""
    randn = rng(D)
    x, w = randn(9, D).to(dt), 1 + randn(D, std=0.1)
    x[1] = 0
    x[2, D // 2], x[3, 1], x[4, D - 1] = float("nan"), float("inf"), float("-inf")
    x[5] *= 1e-30
    x[6] *= 1e-20
    x[7, :] = 0
    x[7, 3] = 1e-30
    for k, eps in ((1.0, 1e-6), (1e-20, 1e-6), (1e-10, 1e-38), (1e25, 1e-6)):
        q, scale = gb.rms_norm(x, w * k, eps=eps, e4m3=True)[:2]
        y = ref.norm(x, w * k, eps)[0]
        want = least_scale(y.float())
        plain = [0, 1, 2, 3, 4, 8]
        assert torch.equal(scale.double()[plain], want[plain]), (k, scale, want)
        got = q.double() * scale.double()[:, None]
        for i in (0, 1, 8):
            assert torch.equal(q[i].float(), (y[i].float().double() / want[i]).float().to(E4M3).float()), (k, i)
        assert bool(got[2].isnan().all()) and bool(got[3, 1].isnan()) and not got[3, 2:].any() and not got[4, :-1].any()
        assert float(scale[2]) == float(scale[3]) == float(scale[4]) == 1
        # the small rows: a half step of e4m3, and what a root of a sum of squares near fp32's least numbers leaves
        a = y[5:8].abs()
        assert bool(((got[5:8] - y[5:8]).abs() <= a * 0.07 + scale[5:8, None].double() * 2.0 ** -10 + 2.0 ** -126).all()), k


def test_e4m3_rows_are_those_of_the_exact_product():
    """Millions of values, equal to the 64-bit form rounded to fp32 and then to e4m3: sums and products in plain fp32 put several of
    them on the other side of a tie. Both forms of y differ by some 2^-46, so that one in 2^22 of the values rounds to
    another fp32 number, and of these the one in 2^20 next to a tie to another e4m3."""
    for T, D, dt in ((8192, 1536, BF), (2048, 1536, F32), (1024, 4096, BF), (300, 16384, F32)):
        randn = rng(T + D)
        x, r, w = randn(T, D).to(dt), randn(T, D, std=2).to(dt), 1 + randn(D, std=0.1)
        q, scale, h, _ = gb.rms_norm(x, w, residual=r, e4m3=True)
        y = ref.norm(h, w, 1e-6)[0].float()
        want = least_scale(y)
        assert torch.equal(scale.double(), want)
        assert torch.equal(q.float(), (y.double() / want[:, None]).float().to(E4M3).float())


@pytest.mark.parametrize("D", [8, 264, 1536, 4096, 8200, 16384])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("residual", [False, True])
def test_e4m3_values_next_to_ties(D, dt, residual):
    """Rows of one magnitude and eps 0: y is w, up to sign, whatever the magnitude. With w at ties of e4m3 and one fp32 number to
    either side, a y that is off by its last place is another e4m3 value."""
    g = torch.Generator(device="cuda").manual_seed(D)
    T = 300
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    h = ((1 + rand(T, 1)) * torch.exp2((rand(T, 1) * 20 - 10).round())).to(dt) * torch.where(rand(T, D) < 0.5, 1, -1).to(dt)
    tie = (17 + 2 * (rand(D) * 8).floor()) / 16 * torch.exp2((rand(D) * 14).floor() - 6)
    tie = torch.where(rand(D) < 0.1, (2 * (rand(D) * 8).floor() + 1) * 2.0 ** -10, tie)
    w = torch.where(rand(D) < 0.34, tie, torch.nextafter(tie, torch.where(rand(D) < 0.5, 0.0, 1000.0)))
    w[0] = 300.0
    q, scale = gb.rms_norm(h, w, residual=torch.zeros_like(h) if residual else None, eps=0.0, e4m3=True)[:2]
    assert bool((scale == 1).all())
    assert torch.equal(q.float(), (h.float().sign() * w).to(E4M3).float())


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_angles_in_fp32(layout, inverse):
    """Pairs (1, 0) become a cosine and a sine. sincospif is within one unit of its last place, 2^-24 below 1; the rest of the angle
    adds a rounding, 2^-25; the angle's own error at positions up to 2^20 (theta's 53 bits, and the reference's angle) is below
    2^20 2^-51. Angles of 24 bits alone would be off by up to 2^-26 of a turn, 2^-23.3."""
    g = torch.Generator(device="cuda").manual_seed(2)
    T, axes, P = 20000, (32, 96), 128
    pos = torch.randint(-2 ** 20, 2 ** 20, (T, 2), generator=g, device="cuda", dtype=torch.int32)
    x = torch.zeros(1, T, 1, 2 * P, device="cuda")
    x[..., 0::2 if layout == "pairs" else 1][..., :P] = 1
    y = gb.rope_axes(x, pos, axes, layout=layout, inverse=inverse)
    want = ref.rope(x, pos, axes, 10000.0, layout, False, inverse)
    near(y, want, torch.full_like(want, 2.0 ** -24 + 2.0 ** -25 + 2.0 ** -30), "angles")


@pytest.mark.parametrize("T,K,N", [(3, 256, 8192), (40, 1536, 6144), (64, 512, 16384), (256, 1536, 1536)])
def test_few_rows_backward_queued(T, K, N):
    """Backward passes of few rows queued far ahead of the GPU: each launches the few-row product early, behind the grid of the
    slopes, and the next slopes behind it."""
    randn = rng(T)
    x, W = randn(T, K).to(BF), randn(N, K, std=K ** -0.5).to(BF)
    Wg = torch.cat((W, W))
    dy, z, zg = randn(T, N).to(BF), randn(T, N).to(BF), randn(T, 2 * N).to(BF)
    want = [gb.linear_backward(dy, x, W, z=z, act="gelu", bias=True), gb.gated_linear_backward(dy, x, Wg, zg), (gb.gated_linear(x, Wg),)]
    for _ in range(150):
        got = [gb.linear_backward(dy, x, W, z=z, act="gelu", bias=True), gb.gated_linear_backward(dy, x, Wg, zg), (gb.gated_linear(x, Wg),)]
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    for a, b in zip(sum(map(list, got), []), sum(map(list, want), [])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dt", [BF, F32])
def test_rope_strides_of_single_rows(layout, dt):
    """A dimension of one has no stride: odd and huge ones there are nothing to a call."""
    randn = rng(7)
    row = randn(2, 193).to(dt)[:1, :192]
    x = row.as_strided((1, 1, 3, 64), (193, 193, 64, 1))
    pos = torch.tensor([[17, 5]], device="cuda", dtype=torch.int32)
    want = gb.rope_axes(x.clone(memory_format=torch.contiguous_format), pos, (16, 16), layout=layout)
    assert torch.equal(gb.rope_axes(x, pos, (16, 16), layout=layout), want)
    for st in ((2 ** 50 + 1, 193, 64, 1), (1, 2 ** 43, 64, 1)):
        z = torch.zeros(192, device="cuda", dtype=dt).as_strided((1, 1, 3, 64), st)
        assert torch.equal(gb.rope_axes(x, pos, (16, 16), layout=layout, out=z), want)
        assert torch.equal(gb.rope_axes(z, pos, (16, 16), layout=layout, inverse=True, out=z, stream=torch.cuda.current_stream()),
                           gb.rope_axes(want, pos, (16, 16), layout=layout, inverse=True))


@pytest.mark.parametrize("T,D", [(40, 1536), (9, 4096), (5, 8200), (3, 16384), (64, 264)])
def test_norm_sums_in_fp32(T, D):
    """fp32 rows to what the kernel's tree of sums allows. A thread adds at most 24 squares, then up to ten sums of threads: 34
    roundings of 2^-24, halved by the root; mean, eps, root and quotient add two, the products of y two more."""
    randn = rng(D)
    x, w = randn(T, D), 1 + randn(D, std=0.2)
    y, _, rstd = gb.rms_norm(x, w)
    yr, k = ref.norm(x, w, 1e-6)
    off = (34 / 2 + 2) * 2.0 ** -24
    near(rstd, k, k * off, "rstd")
    near(y, yr, yr.abs() * (off + 2 * 2.0 ** -24), "y")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D", [264, 1536, 4096])
def test_norm_of_rows_that_are_not_finite(D, dt):
    """NaN and infinities stay in their rows, forward; backward too, but for dw, which sums over the rows."""
    randn = rng(D)
    x, r, w, dy = randn(40, D).to(dt), randn(40, D).to(dt), 1 + randn(D, std=0.1), randn(40, D).to(dt)
    good = gb.rms_norm(x, w, residual=r)
    back = gb.rms_norm_backward(dy, x, w, good[2])
    x[3, 5], r[17, 0], x[30, D - 1] = float("nan"), float("inf"), float("-inf")
    bad = gb.rms_norm(x, w, residual=r)
    rows = torch.ones(40, dtype=torch.bool, device="cuda")
    rows[[3, 17, 30]] = False
    for a, b in zip(bad, good):
        assert torch.equal(a[rows], b[rows])
    assert bool(bad[0][3].isnan().all()) and bool(bad[0][17, 0].isnan()) and not bad[0][17, 1:].any()
    assert float(bad[2][17]) == float(bad[2][30]) == 0 and bool(bad[2][3].isnan())
    dx, dw = gb.rms_norm_backward(dy, x, w, good[2])
    assert torch.equal(dx[rows], back[0][rows]) and bool(dx[3].isnan().all())


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_rope_of_values_that_are_not_finite(layout):
    """A NaN or an infinity reaches its own pair alone."""
    x = rng(4)(1, 6, 5, 64).to(BF)
    pos = torch.arange(12, device="cuda", dtype=torch.int32).view(6, 2) + 1
    good = gb.rope_axes(x, pos, (16, 16), layout=layout)
    x[0, 2, 1, 10], x[0, 4, 3, 63], x[0, 5, 0, 0] = float("nan"), float("inf"), float("-inf")
    bad = gb.rope_axes(x, pos, (16, 16), layout=layout)
    where = torch.zeros_like(x, dtype=torch.bool)
    for t, h, i in ((2, 1, 10), (4, 3, 63), (5, 0, 0)):
        where[0, t, h, i] = where[0, t, h, i ^ 1 if layout == "pairs" else (i + 32) % 64] = True
    assert torch.equal(bad[~where], good[~where]) and not bool(bad[where].isfinite().any())


def test_threads_through_the_native_calls():
    """Layer calls from four threads, each on a stream of its own: the extension lets the interpreter's lock go."""
    work, bad, start = [], [], threading.Barrier(4)
    for i in range(4):
        randn = rng(i)
        T, K, N = (5, 70, 300, 1100)[i], 256 + 64 * i, 144 + 8 * i
        x, r, W, w, b = randn(T, K).to(BF), randn(T, K).to(BF), randn(N, K, std=K ** -0.5).to(BF), 1 + randn(K, std=0.1), randn(N)
        pos = torch.randint(0, 99, (T, 2), device="cuda", dtype=torch.int32)
        dy, axes = randn(T, N).to(BF), (8 + 2 * i, 16)

        def run(x=x, r=r, W=W, w=w, b=b, pos=pos, dy=dy, axes=axes, T=T, K=K):
            y, h, rstd = gb.rms_norm(x, w, residual=r)
            z, pre = gb.linear(y, W, bias=b, act="gelu", pre=True)
            dx, dW, db = gb.linear_backward(dy, y, W, z=pre, act="gelu", bias=True)
            dn, dw = gb.rms_norm_backward(dx, h, w, rstd, dh=r)
            q, s = gb.rms_norm(x, w, e4m3=True)[:2]
            return [y, h, rstd, z, pre, dx, dW, db, dn, dw, q.float(), s, gb.rope_axes(x.view(T, K // 64, 64), pos, axes)]

        work.append((run, run()))
    torch.cuda.synchronize()

    def thread(run, want):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                start.wait()
                for _ in range(200):
                    got = run()
            s.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                bad.append("results differ")
        except Exception as e:
            bad.append(repr(e))

    threads = [threading.Thread(target=thread, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@pytest.mark.parametrize("T,D", [(50000, 64), (20000, 2304), (12000, 4608)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_e4m3_scale_of_more_rows_than_ctas(T, D, dt):
    """A third of the rows at a scale's border (one magnitude a row, so y is w, and the largest w is 448 / 64), some of NaN, and rows of
    zeros between them, where a CTA has several rows."""
    randn = rng(D)
    g = torch.Generator(device="cuda").manual_seed(T)
    w = torch.rand(D, generator=g, device="cuda") * 6
    w[D // 3] = 7.0
    x = randn(T, D).to(dt)
    x[::3] = torch.where(x[::3] < 0, -1, 1) * (1.5 * torch.exp2(torch.arange(0, T, 3, device="cuda") % 20 - 10.0))[:, None].to(dt)
    x[1::7] = 0
    x[5::1001, D - 1] = float("nan")
    q, scale = gb.rms_norm(x, w, eps=1e-30, e4m3=True)[:2]
    y = ref.norm(x, w, 1e-30)[0].float()
    want = least_scale(y)
    assert torch.equal(scale.double(), want)
    assert torch.equal(q.float().nan_to_num(-1.0), (y.double() / want[:, None]).float().to(E4M3).float().nan_to_num(-1.0))
