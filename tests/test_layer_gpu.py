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


SIZES = [(1, 16, 8), (1, 1536, 1528), (7, 4096, 264), (16, 80, 136), (17, 528, 512), (40, 1040, 1000), (64, 64, 64), (100, 512, 640),
         (129, 208, 1528), (256, 1536, 320), (257, 128, 256), (300, 1536, 392), (515, 80, 1544), (2500, 336, 776), (700, 144, 4104)]


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


# ----------------------------------------------------------------------------- as they are used
def test_rows_behind_the_last_stay():
    """Outputs that are the first rows of larger buffers: nothing behind them is written."""
    for T, K, N in ((5, 256, 136), (70, 256, 136), (300, 1536, 392), (2500, 64, 264)):
        randn, x, W, _, _ = operands(T, K, N, False, 3)
        dy, z = randn(T, N).to(BF), randn(T, N).to(BF)
        big = {n: torch.full((T + 9, c), 7.0, device="cuda", dtype=BF) for n, c in (("y", N), ("z", N), ("dx", K), ("h", K), ("g", N))}
        gb.linear(x, W, act="silu", y=big["y"][:T], z=big["z"][:T])
        gb.linear_backward(dy, x, W, z=z, act="silu", dx=big["dx"][:T])
        gb.rms_norm(x, torch.ones(K, device="cuda"), residual=x, h=big["h"][:T])
        gb.gated_linear(x, torch.cat((W, W)), y=big["g"][:T])
        for n, t in big.items():
            assert bool((t[T:] == 7).all()) and not bool((t[:T] == 7).all(1).any()), (n, T)


def test_no_rows():
    x, W, w = torch.zeros(0, 64, device="cuda", dtype=BF), torch.ones(16, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda")
    y, h, rstd = gb.rms_norm(x, w, residual=x)
    assert y.shape == (0, 64) and rstd.shape == (0,)
    assert gb.linear(x, W).shape == (0, 16) and gb.gated_linear(x, W).shape == (0, 8)
    dy = torch.zeros(0, 16, device="cuda", dtype=BF)
    dx, dW, db = gb.linear_backward(dy, x, W, z=dy, act="gelu", bias=True)
    assert dx.shape == (0, 64) and not dW.any() and not db.any()
    dx, dw = gb.rms_norm_backward(x, x, w, rstd)
    assert not dw.any()
    pos = torch.zeros(0, 1, device="cuda", dtype=torch.int32)
    assert gb.rope_axes(x.view(0, 1, 64), pos, (32,)).shape == (0, 1, 64)


def test_python_refusals_on_the_gpu():
    randn, x, W, _, _ = operands(8, 64, 32, False, 1)
    w = torch.ones(64, device="cuda")
    x8, s8 = ref.e4m3_rows(x)
    pos = torch.zeros(8, 1, device="cuda", dtype=torch.int32)
    h = x.view(8, 1, 64)
    for call in (lambda: gb.rms_norm(x, w.double()), lambda: gb.rms_norm(x, w[:32]), lambda: gb.rms_norm(x.T, w), lambda: gb.rms_norm(x, None),
                 lambda: gb.rms_norm(x, w, residual=x[:4]), lambda: gb.rms_norm(x, w, eps=-1.0), lambda: gb.rms_norm(x, w, h=x),
                 lambda: gb.rms_norm(x[:, :60].contiguous(), w[:60]),
                 lambda: gb.linear(x, W.T), lambda: gb.linear(x, W.float()), lambda: gb.linear(x8, W), lambda: gb.linear(x8, W.to(E4M3)),
                 lambda: gb.linear(x, W, x_scale=s8, w_scale=s8), lambda: gb.linear(x, W, act="tanh"), lambda: gb.linear(x, W, bias=w),
                 lambda: gb.linear(x, W, residual=x), lambda: gb.linear(x, W, y=x), lambda: gb.gated_linear(x, W, act=None),
                 lambda: gb.gated_linear(x, W[:31]), lambda: gb.linear_backward(x, x, W), lambda: gb.linear_backward(x[:, :32].contiguous(), x, W, act="silu"),
                 lambda: gb.linear_backward(x[:, :32].contiguous(), x, W, dx=False, dW=False), lambda: gb.linear_backward(x[:, :32].contiguous(), None, W),
                 lambda: gb.rope_axes(h, pos, (33,)), lambda: gb.rope_axes(h, pos, (16, 16)), lambda: gb.rope_axes(h, pos.long(), (32,)),
                 lambda: gb.rope_axes(h, pos, (32,), layout="x"), lambda: gb.rope_axes(h, pos, (32,), base=1.0), lambda: gb.rope_axes(h, pos[:4], (32,)),
                 lambda: gb.rope_axes(h, pos, (32,), out=h[:1].expand(8, 1, 64)), lambda: gb.rope_axes(h.transpose(0, 2), pos, (32,))):
        with pytest.raises(api.SsbaError):
            call()


def test_short_and_long_way_are_one():
    """Calls that take the native way and calls with their outputs given, on the current and on another stream."""
    randn, x, W, _, _ = operands(70, 256, 144, False, 5)
    w, r, b = 1 + randn(256, std=0.1), randn(70, 256).to(BF), randn(144)
    dy, z = randn(70, 144).to(BF), randn(70, 144).to(BF)
    pos = torch.randint(0, 99, (70, 2), device="cuda", dtype=torch.int32)
    st = torch.cuda.Stream()

    def run(**kw):
        out = [*gb.rms_norm(x, w, residual=r, **kw), *gb.rms_norm(x, w, e4m3=True, **kw)[:2]]
        out += gb.rms_norm_backward(r, x, w, out[2], dh=r, **kw)
        out += [gb.linear(x, W, bias=b, act="gelu", **kw), *gb.linear(x, W, pre=True, **kw), *gb.gated_linear(x, W, pre=True, **kw)]
        out += gb.linear_backward(dy, x, W, z=z, act="silu", bias=True, **kw)
        out += gb.gated_linear_backward(dy[:, :72].contiguous(), x, W, z, **kw)
        out.append(gb.rope_axes(x.view(70, 4, 64), pos, (16, 16), **kw))
        return out

    a, b_ = run(), run(stream=torch.cuda.current_stream())
    st.wait_stream(torch.cuda.current_stream())
    c = run(stream=st)
    with torch.cuda.stream(st):
        d = run()
    torch.cuda.synchronize()
    for i, (p, q, s, t) in enumerate(zip(a, b_, c, d)):
        assert torch.equal(p.float(), q.float()) and torch.equal(p.float(), s.float()) and torch.equal(p.float(), t.float()), i


def layer_forward(desc, p, x, pos, lists=None):
    """One pre-norm layer: norm, projection, rotary positions, sparse attention, projection with residual, norm, gated block.
    Returns every stage."""
    B, N, H = desc.B, desc.N, desc.heads
    s = {}
    s["y1"], _, s["k1"] = gb.rms_norm(x, p["n1"])
    qkv = s["qkv"] = gb.linear(s["y1"], p["Wqkv"], bias=p["b"])
    v5 = qkv.view(B, N, 3, H, 64)
    s["Q"], s["K"], s["V"] = (torch.empty(B, H, N, 64, device="cuda", dtype=BF) for _ in range(3))
    gb.rope_axes(v5[:, :, 0], pos, (16, 16), out=s["Q"].transpose(1, 2))
    gb.rope_axes(v5[:, :, 1], pos, (16, 16), out=s["K"].transpose(1, 2))
    s["V"].copy_(v5[:, :, 2].transpose(1, 2))
    s["O"], s["lse"], s["idx"], s["cnt"] = gb.forward_fused(desc, s["Q"], s["K"], s["V"])[:4]
    s["o"] = s["O"].transpose(1, 2).reshape(B * N, H * 64)
    s["a"] = gb.linear(s["o"], p["Wo"])
    s["y2"], s["h"], s["k2"] = gb.rms_norm(s["a"], p["n2"], residual=x)
    s["g"], s["z"] = gb.gated_linear(s["y2"], p["Wgu"], pre=True)
    s["out"] = gb.linear(s["g"], p["Wd"], residual=s["h"])
    return s


def layer_backward(desc, p, x, pos, s, dout):
    B, N, H = desc.B, desc.N, desc.heads
    g = {}
    dg, g["Wd"], _ = gb.linear_backward(dout, s["g"], p["Wd"])
    dy2, g["Wgu"] = gb.gated_linear_backward(dg, s["y2"], p["Wgu"], s["z"])
    da, g["n2"] = gb.rms_norm_backward(dy2, s["h"], p["n2"], s["k2"], dh=dout)  # of a and, as it is, of x
    do, g["Wo"], _ = gb.linear_backward(da, s["o"], p["Wo"])
    dO = do.view(B, N, H, 64).transpose(1, 2).contiguous()
    dQ, dK, dV = gb.backward(desc, s["Q"], s["K"], s["V"], s["O"], s["lse"], dO, s["idx"], s["cnt"])
    dqkv = torch.empty(B, N, 3, H, 64, device="cuda", dtype=BF)
    gb.rope_axes(dQ.to(BF).transpose(1, 2), pos, (16, 16), inverse=True, out=dqkv[:, :, 0])
    gb.rope_axes(dK.to(BF).transpose(1, 2), pos, (16, 16), inverse=True, out=dqkv[:, :, 1])
    dqkv[:, :, 2].copy_(dV.transpose(1, 2))
    dy1, g["Wqkv"], g["b"] = gb.linear_backward(dqkv.view(B * N, -1), s["y1"], p["Wqkv"], bias=True)
    g["x"], g["n1"] = gb.rms_norm_backward(dy1, x, p["n1"], s["k1"], dh=da)
    return g


def layer_inputs(seed=0, H=2, side=16, F=192):
    randn = rng(seed)
    D = H * 64
    desc = api.SsbaDesc(1, H, side, side, rho=0.5)
    mat = lambda n, k: (randn(n, k) / k ** 0.5).to(BF)  # noqa: E731
    p = dict(n1=1 + randn(D, std=0.1), Wqkv=mat(3 * D, D), b=randn(3 * D, std=0.1), Wo=mat(D, D), n2=1 + randn(D, std=0.1), Wgu=mat(2 * F, D), Wd=mat(D, F))
    n = torch.arange(side * side, device="cuda", dtype=torch.int32)
    return desc, p, randn(side * side, D).to(BF), torch.stack((n // side, n % side), 1), randn(side * side, D, std=0.1).to(BF)


def test_a_layer_forward_and_backward():
    """A layer and its gradients against the whole layer in 64 bits with autograd, on the kernel's lists. Every stage rounds
    to bf16 (2^-9 of its values, on average over sqrt(3)); some twenty of them in a row, each with a gain of about one,
    stay below 20 * 2^-9 = 2^-4.7 of the results' norm."""
    desc, p, x, pos, dout = layer_inputs()
    s = layer_forward(desc, p, x, pos)
    g = layer_backward(desc, p, x, pos, s, dout)
    N, H = desc.N, desc.heads
    d = {k: v.double().requires_grad_(True) for k, v in {**p, "x": x}.items()}
    norm = lambda h, w: h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w  # noqa: E731
    qkv = (norm(d["x"], d["n1"]) @ d["Wqkv"].T + d["b"]).view(1, N, 3, H, 64)
    th = 10000.0 ** (-torch.arange(16, device="cuda", dtype=torch.float64) / 16)
    ang = torch.cat((pos[:, :1].double() * th, pos[:, 1:].double() * th), 1)[None, :, None]
    def turn(t):
        u, v = t[..., 0::2], t[..., 1::2]
        return torch.stack((u * ang.cos() - v * ang.sin(), u * ang.sin() + v * ang.cos()), -1).flatten(-2)
    Q, K, V = turn(qkv[:, :, 0]).transpose(1, 2), turn(qkv[:, :, 1]).transpose(1, 2), qkv[:, :, 2].transpose(1, 2)
    label = (torch.arange(N, device="cuda") // 16 // 8) * 2 + (torch.arange(N, device="cuda") % 16) // 8
    kept = torch.zeros(1, H, 4, 4, device="cuda").scatter_(3, s["idx"].long(), 1.0) > 0
    mask = kept[:, :, label][:, :, :, label]
    a = (Q @ K.transpose(2, 3) / 8).masked_fill(~mask, float("-inf")).softmax(3) @ V
    h = a.transpose(1, 2).reshape(N, H * 64) @ d["Wo"].T + d["x"]
    z = norm(h, d["n2"]) @ d["Wgu"].T
    F = z.shape[1] // 2
    out = (torch.nn.functional.silu(z[:, :F]) * z[:, F:]) @ d["Wd"].T + h
    grads = torch.autograd.grad(out, list(d.values()), dout.double())
    far = lambda got, want: float((got.double() - want.detach()).norm() / want.detach().norm())  # noqa: E731
    assert far(s["out"], out) < 2.0 ** -4.7
    for name, want in zip(d, grads):
        assert far(g[name], want) < 2.0 ** -4.7, name


def test_a_layer_in_two_graphs():
    """Forward and backward of a layer captured twice, replayed in turn on new inputs, with eager calls between."""
    desc, p, x, pos, dout = layer_inputs(1)
    st = torch.cuda.Stream()
    state = []
    for seed in (1, 2):
        _, _, xi, _, di = layer_inputs(seed)
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            layer_backward(desc, p, xi, pos, layer_forward(desc, p, xi, pos), di)
        torch.cuda.current_stream().wait_stream(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s = layer_forward(desc, p, xi, pos)
            g = layer_backward(desc, p, xi, pos, s, di)
        state.append((graph, xi, di, s, g))
    for round_ in range(3):
        for i, (graph, xi, di, s, g) in enumerate(state):
            _, _, nx, _, nd = layer_inputs(10 + 2 * round_ + i)
            xi.copy_(nx)
            di.copy_(nd)
        for graph, *_ in state:
            graph.replay()
        for graph, xi, di, s, g in state:
            e = layer_forward(desc, p, xi, pos)
            eg = layer_backward(desc, p, xi, pos, e, di)
            torch.cuda.synchronize()
            assert torch.equal(s["out"], e["out"])
            for n in eg:
                assert torch.equal(g[n], eg[n]), n


def test_many_calls_queued():
    """Backward passes queued far ahead of the GPU, as a training loop leaves them, and chains of few-token calls."""
    randn, x, W, _, _ = operands(1500, 512, 1024, False, 9, 2048)
    dy, z = randn(1500, 1024).to(BF), randn(1500, 2048).to(BF)
    want = gb.gated_linear_backward(dy, x, W, z)
    few = x[:8].contiguous()
    first = gb.linear(gb.gated_linear(few, W), W[:512, :].reshape(256, 1024))
    for i in range(300):
        dx, dW = gb.gated_linear_backward(dy, x, W, z)
        y, _, _ = gb.rms_norm(dx, torch.ones(512, device="cuda"))
        a = gb.linear(gb.gated_linear(few, W), W[:512, :].reshape(256, 1024))
    torch.cuda.synchronize()
    assert torch.equal(dx, want[0]) and torch.equal(dW, want[1]) and torch.equal(a, first)


def test_past_32_bits():
    """Rows whose offsets pass 2^31 elements, and 2^32 bytes."""
    T, D = 540000, 4096
    x = torch.zeros(T, D, device="cuda", dtype=BF)
    x[-40:] = torch.randn(40, D, device="cuda").to(BF)
    w = torch.ones(D, device="cuda")
    y, _, k = gb.rms_norm(x, w)
    yr, kr = ref.norm(x[-40:], w, 1e-6)
    near(y[-40:], yr, yr.abs() * (2.0 ** -8 + 2.0 ** -10))
    assert not y[:-40].any()
    dx, dw = gb.rms_norm_backward(x, x, w, k)
    want, _ = ref.norm_backward(x[-40:], x[-40:], w, k[-40:], None)
    near(dx[-40:], want, want.abs() * 2.0 ** -8 + 2.0 ** -10)
    del y, dx
    W = (torch.randn(D, 64, device="cuda") / 8).to(BF)
    r = x[:, :64].contiguous()
    out = gb.linear(r, W)  # [T, 4096]
    yr, _, ty, _ = ref.linear(r[-40:], W)
    near(out[-40:], yr, ty)
    assert not out[:-40].any()
    pos = torch.zeros(T, 1, device="cuda", dtype=torch.int32)
    pos[-40:] = 5
    turned = gb.rope_axes(x.view(T, 64, 64), pos, (32,), layout="halves", out=out.view(T, 64, 64))
    near(turned[-40:], ref.rope(x[-40:].view(1, 40, 64, 64), pos[-40:], (32,), layout="halves")[0], 0.05 + 0 * turned[-40:].double())


def test_more_rows_than_a_grid_has():
    """Narrow products of nine million rows: the few-row kernel's grid would not hold them."""
    T = 9 * 2 ** 20
    x = torch.zeros(T, 8, device="cuda", dtype=BF)
    x[-5:] = torch.randn(5, 8, device="cuda").to(BF)
    W = torch.randn(8, 8, device="cuda").to(BF)
    y = gb.linear(x, W)
    yr, _, ty, _ = ref.linear(x[-5:], W)
    near(y[-5:], yr, ty)
    assert not y[:-5].any()
    dx, dW, _ = gb.linear_backward(x, x, W)
    want = ref.linear_backward(x[-5:], x[-5:], W, None, None)
    near(dx[-5:], *want[0])
    near(dW, *want[1])


@pytest.mark.parametrize("T,K,N", [(5000, 72, 64), (9000, 520, 264), (20000, 1536, 392)])
def test_weights_gradient_of_many_tokens(T, K, N):
    """Few tiles and a long sum: dW is summed in parts. Alone and beside dx it is the same."""
    randn, x, W, _, _ = operands(T, K, N, False, T)
    dy, z = randn(T, N).to(BF), randn(T, N, std=2).to(BF)
    for act in (None, "silu"):
        zz = z if act else None
        got = gb.linear_backward(dy, x, W, z=zz, act=act, bias=True)
        for g, (want, tol), what in zip(got, ref.linear_backward(dy, x, W, zz, act), ("dx", "dW", "db")):
            near(g, want, tol, what)
        assert torch.equal(gb.linear_backward(dy, x, None, z=zz, act=act, dx=False)[1], got[1])
        into = torch.zeros_like(got[1])
        ws = torch.zeros(gb.linear_backward_workspace_bytes(T, N, K, act), dtype=torch.uint8, device="cuda")
        gb.linear_backward(dy, x, W, z=zz, act=act, dW=into, workspace=ws)
        assert torch.equal(into, got[1])


@pytest.mark.parametrize("T,K,N", [(5, 4096, 256), (40, 64, 136), (100, 512, 640), (2500, 336, 776), (9000, 512, 1536)])
@pytest.mark.parametrize("is_gated", [False, True])
def test_a_wait_that_runs_out(T, K, N, is_gated):
    """Copies that never come: every kernel gives up, says so, and the next call is right."""
    from paper_2605_15684_gb300 import layer
    _, x, W, _, _ = operands(T, K, N, False, 4, 2 * N if is_gated else N)
    call = gb.gated_linear if is_gated else gb.linear
    want = call(x, W)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK
    layer.test_linear_timeout(x, W, torch.empty_like(want), gated=is_gated, budget_ns=3_000_000)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_ERR_TIMEOUT
    assert torch.equal(call(x, W), want)
    torch.cuda.synchronize()
    assert api.get_status() == api.SSBA_OK


def test_sums_at_odd_addresses():
    """dw and db that are 4-byte aligned only, of few rows (whose sums are written without a join) and of many."""
    for T in (3, 100, 700):
        randn, x, W, _, _ = operands(T, 64, 72, False, T)
        dy, z, w = randn(T, 72).to(BF), randn(T, 72).to(BF), 1 + randn(64, std=0.1)
        _, _, rstd = gb.rms_norm(x, w)
        dx, dw = gb.rms_norm_backward(x, x, w, rstd)
        db = gb.linear_backward(dy, x, W, z=z, act="gelu", bias=True)[2]
        odd = torch.zeros(138, device="cuda")
        gb.rms_norm_backward(x, x, w, rstd, dw=odd[1:65])
        gb.linear_backward(dy, x, W, z=z, act="gelu", db=odd[65:137])
        assert torch.equal(odd[1:65], dw) and torch.equal(odd[65:137], db) and not odd[0] and not odd[137]


def test_norm_of_tiny_rows_without_eps():
    """eps 0 and rows of 1e-15 (rstd 1e15) and of 1e15: the gradient neither overflows nor vanishes on the way."""
    randn = rng(8)
    h = randn(6, 264) * torch.tensor([1e-15, 1e15, 1.0, 1e-12, 1e10, 3.0], device="cuda")[:, None]
    w, dy = 1 + randn(264, std=0.1), randn(6, 264)
    for dt in (BF, F32):
        hh, dd = h.to(dt), dy.to(dt)
        y, _, rstd = gb.rms_norm(hh, w, eps=0.0)
        yr, k = ref.norm(hh, w, 0.0)
        near(y, yr, yr.abs() * (ref.half_step(dt) + 2.0 ** -14))
        dx, dw = gb.rms_norm_backward(dd, hh, w, rstd)
        want, wdw = ref.norm_backward(dd, hh, w, k, None)
        size = (dd.double() * w.double()).abs().amax(1, keepdim=True) * k[:, None]
        near(dx, want, want.abs() * ref.half_step(dt) + size * 2.0 ** -14, "dx")
        near(dw, wdw, (dd.double().abs() * (hh.double() * k[:, None]).abs()).sum(0) * 2.0 ** -14, "dw")


def test_two_streams_at_once():
    """Products of both kernels on one stream while rows of many waves of CTAs, and other products, run on another."""
    randn, x, W, _, _ = operands(3000, 512, 1024, False, 9, 2048)
    dy, z, w = randn(3000, 1024).to(BF), randn(3000, 2048).to(BF), torch.ones(512, device="cuda")
    rows = randn(60000, 512).to(BF)
    few = x[:9].contiguous()

    def a():
        return [*gb.gated_linear_backward(dy, x, W, z), gb.linear(x, W), gb.gated_linear(few, W)]

    def b():
        return [gb.rms_norm(rows, w)[0], gb.linear(few, W), gb.linear(rows, W[:256].contiguous()), gb.gated_linear(x, W)]

    want_a, want_b = a(), b()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(30):
        with torch.cuda.stream(s):
            got_a = a()
        with torch.cuda.stream(t):
            got_b = b()
    torch.cuda.synchronize()
    for got, want in zip(got_a + got_b, want_a + want_b):
        assert torch.equal(got, want)
