"""GPU parity of a layer's operators (rms_norm, linear, gated_linear, rope_axes and their gradients) with plain 64-bit
forms, at the sizes and layouts where they change paths or could go wrong. Tolerances: layer_ref.py."""
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


# ----------------------------------------------------------------------------- the norm
@pytest.mark.parametrize("T,D", [(1, 8), (3, 256), (1, 1536), (37, 264), (301, 1536), (65, 1544), (5, 2048), (33, 2056), (9, 4096),
                                 (7, 8184), (2, 8200), (3, 16384)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
def test_norm(T, D, dt, residual, e4m3):
    randn = rng(T * 31 + D)
    x, r, w = randn(T, D).to(dt), randn(T, D, std=3).to(dt) if residual else None, 1 + randn(D, std=0.2)
    out = gb.rms_norm(x, w, residual=r, e4m3=e4m3)
    h, rstd = out[-2:]
    if residual:
        near(h, x.double() + r.double(), (x.double() + r.double()).abs() * ref.half_step(dt), "h")
    else:
        assert h is x
    y, k = ref.norm(h, w, 1e-6)
    # the mean: D squares and sums of 2^-24 each, halved by the root; then root and quotient
    off = (D * 2.0 ** -24 + 2.0 ** -22)
    near(rstd, k, k * off, "rstd")
    if not e4m3:
        near(out[0], y, y.abs() * (ref.half_step(dt) + 2 * off), "y")
        return
    q, scale = out[:2]
    assert q.dtype == E4M3 and bool((scale.log2() == scale.log2().round()).all())
    a = y.abs().amax(1) / scale.double()
    assert bool((a <= 448 * (1 + 2 * off)).all()) and bool((a > 224 * (1 - 2 * off)).all())
    s = scale.double()[:, None]
    near(q.double() * s, y, y.abs() * (2.0 ** -4 + 2 * off) + s * 2.0 ** -10, "e4m3 rows")


def test_norm_special_rows():
    """A row of zeros, one of tiny and one of huge values, in 8 bits and in bf16; and outputs on top of inputs."""
    x = torch.zeros(4, 64, device="cuda", dtype=BF)
    x[1], x[2, 0], x[3] = 1e-20, 2.0 ** 60, -3.0
    w = torch.ones(64, device="cuda")
    q, s, h, rstd = gb.rms_norm(x, w, eps=1e-6, e4m3=True)
    assert float(s[0]) == 1 and not q[0].float().any()
    y, k = ref.norm(x, w, 1e-6)
    near(q.double() * s.double()[:, None], y, y.abs() * 0.07 + s.double()[:, None] * 2.0 ** -10)
    y0, _, _ = gb.rms_norm(x, w)
    x2 = x.clone()
    y2, _, _ = gb.rms_norm(x2, w, y=x2)
    assert y2 is x2 and torch.equal(y2, y0)
    r = torch.randn(4, 64, device="cuda").to(BF)
    y3, h3, _ = gb.rms_norm(x, w, residual=r)
    r2 = r.clone()
    y4, h4, _ = gb.rms_norm(x, w, residual=r2, h=r2)
    assert h4 is r2 and torch.equal(h4, h3) and torch.equal(y4, y3)


@pytest.mark.parametrize("T,D", [(1, 8), (5, 256), (301, 264), (2000, 1536), (33, 2048), (700, 4096), (9, 8200), (3, 16384)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("dh", [False, True])
def test_norm_backward(T, D, dt, dh):
    randn = rng(T + D)
    h, dy, w = randn(T, D).to(dt), randn(T, D).to(dt), 1 + randn(D, std=0.2)
    g = randn(T, D).to(dt) if dh else None
    _, k = ref.norm(h, w, 1e-5)
    rstd = k.float()
    dx, dw = gb.rms_norm_backward(dy, h, w, rstd, dh=g)
    dxr, dwr = ref.norm_backward(dy, h, w, k, g)
    xh, gw = h.double() * k[:, None], dy.double() * w.double()
    along = (gw * xh).abs().mean(1, keepdim=True)
    terms = k[:, None] * (gw.abs() + xh.abs() * along)
    e = terms * (D + 16) * 2.0 ** -24
    near(dx, dxr, e + (dxr.abs() + e) * (ref.half_step(dt) + 2.0 ** -23), "dx")
    near(dw, dwr, (dy.double() * xh).abs().sum(0) * (T + 16) * 2.0 ** -24 + 1e-30, "dw")
    again = gb.rms_norm_backward(dy, h, w, rstd, dh=g)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])  # one order of every sum
    if dh:
        into, _ = gb.rms_norm_backward(dy, h, w, rstd, dh=g, dx=g)
        assert into is g and torch.equal(into, dx)


# ----------------------------------------------------------------------------- products
def operands(T, K, N, f8, seed, rows=None):
    randn = rng(seed)
    x, W = randn(T, K), randn(rows or N, K, std=K ** -0.5)
    if f8:
        (x, xs), (W, ws) = ref.e4m3_rows(x * torch.exp(randn(T, 1))), ref.e4m3_rows(W)
        return randn, x, W, xs, ws
    return randn, x.to(BF), W.to(BF), None, None


SIZES = [(1, 16, 8), (1, 1536, 1536), (7, 4096, 264), (16, 80, 136), (17, 528, 512), (40, 1040, 1000), (64, 64, 64), (100, 512, 640),
         (129, 208, 1536), (256, 1536, 320), (257, 128, 256), (300, 1536, 392), (515, 80, 1544), (2500, 336, 776), (700, 144, 4104)]


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("act,bias,residual,pre", [(None, False, False, False), ("gelu", True, False, True), ("silu", True, True, False),
                                                   ("relu", False, True, True)])
def test_linear(T, K, N, f8, act, bias, residual, pre):
    randn, x, W, xs, ws = operands(T, K, N, f8, T + K + N)
    b = randn(N) if bias else None
    r = randn(T, N).to(BF) if residual else None
    out = gb.linear(x, W, bias=b, residual=r, act=act, x_scale=xs, w_scale=ws, pre=pre)
    y, z = out if pre else (out, None)
    yr, zr, ty, tz = ref.linear(x, W, b, r, act, xs, ws)
    near(y, yr, ty, "y")
    if pre:
        near(z, zr, tz + (zr.abs() + tz) * 2.0 ** -8, "z")
        assert torch.equal(gb.linear(x, W, bias=b, residual=r, act=act, x_scale=xs, w_scale=ws), y)
    if residual:
        into = gb.linear(x, W, bias=b, residual=r, act=act, x_scale=xs, w_scale=ws, y=r)
        assert into is r and torch.equal(into, y)


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("act,pre", [("silu", False), ("gelu", True), ("relu", False)])
def test_gated(T, K, N, f8, act, pre):
    randn, x, W, xs, ws = operands(T, K, N, f8, T + K + N, 2 * N)
    out = gb.gated_linear(x, W, act=act, x_scale=xs, w_scale=ws, pre=pre)
    y, z = out if pre else (out, None)
    yr, zr, ty, tz = ref.gated(x, W, act, xs, ws)
    near(y, yr, ty, "y")
    if pre:
        near(z, zr, tz + (zr.abs() + tz) * 2.0 ** -8, "z")
        assert torch.equal(gb.gated_linear(x, W, act=act, x_scale=xs, w_scale=ws), y)


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("act,bias", [(None, False), (None, True), ("gelu", True), ("silu", False), ("relu", True)])
def test_linear_backward(T, K, N, act, bias):
    randn, x, W, _, _ = operands(T, K, N, False, T + K + N)
    dy, z = randn(T, N).to(BF), randn(T, N, std=2).to(BF) if act else None
    got = gb.linear_backward(dy, x, W, z=z, act=act, bias=bias)
    want = ref.linear_backward(dy, x, W, z, act)
    near(got[0], *want[0], "dx")
    near(got[1], *want[1], "dW")
    if bias:
        near(got[2], *want[2], "db")
    else:
        assert got[2] is None
    dx, none, _ = gb.linear_backward(dy, None, W, z=z, act=act, dW=False)
    assert none is None and torch.equal(dx, got[0])
    none, dW, db = gb.linear_backward(dy, x, None, z=z, act=act, dx=False, bias=bias)
    assert none is None and torch.equal(dW, got[1]) and (db is None or torch.equal(db, got[2]))


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gated_backward(T, K, N, act):
    randn, x, W, _, _ = operands(T, K, N, False, T + K + N, 2 * N)
    dy, z = randn(T, N).to(BF), randn(T, 2 * N, std=2).to(BF)
    dx, dW = gb.gated_linear_backward(dy, x, W, z, act=act)
    want = ref.linear_backward(dy, x, W, z, act, True)
    near(dx, *want[0], "dx")
    near(dW, *want[1], "dW")


def test_activations_at_the_ends():
    """Arguments where exponentials overflow and slopes vanish, and NaN and infinities in their own rows alone."""
    z = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 5, -5, 20, -20, 88, -88, 100, -100, 1e4, -1e4, 3e38, -3e38], device="cuda")
    W = torch.eye(16, device="cuda").to(BF)
    x = z.to(BF)[None].repeat(3, 1)
    for act in ("relu", "gelu", "silu"):
        for n in (3, 300):  # both kernels
            got = gb.linear(x[:1].repeat(n, 1), W[:, :16], act=act)
            yr = ref.act(x[:1].double(), act)
            near(got, yr.repeat(n, 1), yr.abs().repeat(n, 1) * (2.0 ** -8 + 2.0 ** -15) + 1e-30, act)
        dy = torch.ones(1, 16, device="cuda", dtype=BF)
        dx, _, db = gb.linear_backward(dy, x[:1], W, z=x[:1], act=act, bias=True)
        want = ref.slope(x[:1], act, False, dy)
        near(db[None], want, torch.full_like(want, 2.0 ** -14), act)
    bad = torch.randn(300, 64, device="cuda").to(BF)
    W = torch.randn(64, 64, device="cuda").to(BF)
    good = gb.linear(bad, W, act="silu")
    bad[7, 3], bad[200, 0] = float("nan"), float("inf")
    y = gb.linear(bad, W, act="silu")
    rows = torch.ones(300, dtype=torch.bool, device="cuda")
    rows[[7, 200]] = False
    assert torch.equal(y[rows], good[rows]) and bool(y[7].isnan().all())


# ----------------------------------------------------------------------------- rotary positions
ROPE = [
    (1, 1, 1, 64, (32,), "pairs"), (2, 5, 3, 64, (16, 16), "pairs"), (1, 300, 24, 64, (16, 16), "halves"),
    (3, 7, 2, 128, (16, 24, 24), "halves"), (1, 33, 8, 96, (7, 11, 5), "pairs"), (1, 33, 8, 96, (7, 11, 5), "halves"),
    (2, 40, 4, 80, (12, 4, 4, 8), "halves"), (1, 17, 5, 256, (128,), "halves"), (1, 64, 1, 6, (1, 1), "pairs"), (1, 64, 3, 6, (2,), "halves"),
]


@pytest.mark.parametrize("B,T,H,D,axes,layout", ROPE)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("shared,inverse", [(False, False), (True, True)])
def test_rope(B, T, H, D, axes, layout, dt, shared, inverse):
    randn = rng(B + T + D)
    x = randn(B, T, H, D).to(dt)
    g = torch.Generator(device="cuda").manual_seed(5)
    for pos in (torch.randint(-50, 2000, (T, len(axes)), generator=g, device="cuda", dtype=torch.int32),
                torch.randint(-2 ** 31, 2 ** 31 - 1, (B, T, len(axes)), generator=g, device="cuda", dtype=torch.int32)):
        y = gb.rope_axes(x, pos, axes, layout=layout, shared=shared, inverse=inverse)
        want = ref.rope(x, pos, axes, 10000.0, layout, shared, inverse)
        # the reference's angle (a 64-bit product, then a cosine of it) is off by 2^-52 of up to 2^31 radians; the kernel's
        # by 2^-32 of a turn, and sine and cosine by 2^-22; each element is a sum of two products
        P = sum(axes)
        p = x.double().abs()
        pair = p.clone()
        u, v = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "pairs" else (slice(0, P), slice(P, 2 * P))
        pair[..., u] = pair[..., v] = p[..., u] + p[..., v]
        near(y, want, pair * (2.0 ** -20 + 2.0 ** -21) + want.abs() * ref.half_step(dt), "rope")
        assert torch.equal(y[..., 2 * P:], x[..., 2 * P:])


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dt", [BF, F32])
def test_rope_strides(layout, dt):
    """Parts of a packed projection, head-major outputs, in place, rows that allow no wide access, 3-D calls."""
    B, T, H, D, axes = 2, 19, 3, 64, (8, 12, 12)
    randn = rng(3)
    qkv = randn(B, T, 3, H, D).to(dt)
    pos = torch.randint(0, 90, (T, 3), device="cuda", dtype=torch.int32)
    want = gb.rope_axes(qkv[:, :, 1].contiguous(), pos, axes, layout=layout)
    near(want, ref.rope(qkv[:, :, 1], pos, axes, layout=layout), 0.02 + 0 * want.double())
    out = torch.empty(B, H, T, D, device="cuda", dtype=dt)
    gb.rope_axes(qkv[:, :, 1], pos, axes, layout=layout, out=out.transpose(1, 2))
    assert torch.equal(out.transpose(1, 2), want)
    rest = qkv.clone()
    gb.rope_axes(qkv[:, :, 1], pos, axes, layout=layout, out=qkv[:, :, 1])
    assert torch.equal(qkv[:, :, 1], want) and torch.equal(qkv[:, :, 0], rest[:, :, 0]) and torch.equal(qkv[:, :, 2], rest[:, :, 2])
    odd = 2 if layout == "pairs" else 1
    wide = torch.zeros(B, T, H, D + odd, device="cuda", dtype=dt)
    wide[..., odd:] = rest[:, :, 1]
    got = gb.rope_axes(wide[..., odd:], pos, axes, layout=layout, out=wide[..., odd:])
    assert torch.equal(got, want) and not wide[..., :odd].any()
    one = gb.rope_axes(rest[0, :, 1], pos, axes, layout=layout)
    assert one.dim() == 3 and torch.equal(one, want[0])
    back = gb.rope_axes(want, pos, axes, layout=layout, inverse=True)
    near(back, rest[:, :, 1].double(), torch.full_like(back, 0.05 if dt == BF else 1e-5).double())


def test_rope_is_the_projections():
    """The 2-D positions of qkv_rope_pool: 16 pairs of the token's row, 16 of its column."""
    from paper_2605_15684_gb300 import synthetic
    X, Wq, b = synthetic.projection_inputs(1, 256, 128, 3)
    desc = api.SsbaDesc(1, 2, 16, 16, rho=0.5)
    Q, K, V, _, _ = api.qkv_rope_pool(desc, X.cuda(), Wq.cuda(), b.cuda(), pooled=False)
    qkv = gb.linear(X[0].cuda(), Wq.cuda(), bias=b.cuda()).view(1, 256, 3, 2, 64)
    n = torch.arange(256, device="cuda", dtype=torch.int32)
    pos = torch.stack((n // 16, n % 16), 1)
    for i, want in ((0, Q), (1, K)):
        got = gb.rope_axes(qkv[:, :, i], pos, (16, 16)).transpose(1, 2)
        # one rounding more here: of the projection, a pair's two
        near(got, want.double(), 2.0 ** -7 * want.double().abs() + 2.0 ** -7 * 6)
    assert float((qkv[:, :, 2].transpose(1, 2).double() - V.double()).abs().max()) <= 2.0 ** -7 * float(V.abs().max())
