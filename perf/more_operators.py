"""The work of a transformer layer around its attention: the root-mean-square norm with the residual's
addition (16-bit rows, or 8-bit rows with scales), products with weights and what follows them in the
same pass (bias, activation, residual), the gated half of a feed-forward block, and rotary positions
with several axes, for prompts and images, for single tokens, and backward.

Rows are tokens, in any number; widths are multiples of 16. 8-bit values are e4m3 with one
power-of-two scale a row, and are returned as the values they stand for.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
BF16, FP32, F8 = "bf16", "fp32", "e4m3"
_DT = {BF16: torch.bfloat16, FP32: torch.float32}
EPS = 1e-6


# ----------------------------------------------------------------------------- the cases
def listed():
    return [
        # One token of a served model: the smallest call.
        dict(op="norm", T=1, D=1536, dtype=BF16, out=BF16, residual=True, name="norm_token"),
        # The tokens of a 1024 px image, a layer of this library's 24 heads of 64, in front of an 8-bit product.
        dict(op="norm", T=4096, D=1536, dtype=BF16, out=F8, residual=True, name="norm_image_e4m3"),
        # Training on long rows, an odd number of tokens; the residual's own gradient joins.
        dict(op="norm_bwd", T=16001, D=4096, dtype=BF16, residual=True, name="norm_backward_16k"),
        # Seven tokens through the projection behind the attention: weights are read once for all.
        dict(op="linear", T=7, K=4096, N=4096, dtype=BF16, bias=True, act="none", residual=True, name="linear_7_tokens"),
        # The first product of a plain feed-forward block on four 1024 px images, 8-bit operands.
        dict(op="linear", T=16384, K=1536, N=6144, dtype=F8, bias=True, act="gelu", residual=False, name="linear_ffn_e4m3"),
        # Backward of the same product in 16 bits for one image and its text tokens (4096 + 77).
        dict(op="linear_bwd", T=4173, K=1536, N=6144, dtype=BF16, bias=True, act="gelu", residual=False, name="linear_backward_4k"),
        # The gated block's projections for 32 sequences' single tokens in 8 bits.
        dict(op="gated", T=32, K=4096, F=12288, dtype=F8, act="silu", name="gated_32_tokens_e4m3"),
        # A batch of prompts, 16-bit operands: the largest product.
        dict(op="gated", T=8192, K=4096, F=12288, dtype=BF16, act="silu", name="gated_8k"),
        # A training step's backward through the gated projections, an odd number of rows.
        dict(op="gated_bwd", T=5001, K=2048, F=5632, dtype=BF16, act="silu", name="gated_backward_5k"),
        # One token each of 16 sequences, far along: adjacent pairs, one position.
        dict(op="rope", B=16, T=1, heads=32, d=128, axes="64", layout="halves", shared=True, far=1000000, dtype=BF16, inverse=False, name="rope_tokens_far"),
        # Queries of a 1024 px image out of the packed projection, into the attention's head-major layout.
        dict(op="rope", B=1, T=4096, heads=24, d=64, axes="16,16", layout="pairs", shared=False, far=64, dtype=BF16, inverse=False, name="rope_image"),
        # A video's gradient turned back: time, height and width, 41 frames of 45 x 26 tokens.
        dict(op="rope", B=1, T=47970, heads=24, d=128, axes="16,24,24", layout="halves", shared=True, far=64, dtype=BF16, inverse=True, name="rope_video_backward"),
    ]


def _log(rng, lo, hi):
    return max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    """One more case: the same operators over their whole ranges, none larger than the largest listed."""
    while True:
        op = rng.choice(["norm", "norm_bwd", "linear", "linear", "linear_bwd", "gated", "gated", "gated_bwd", "rope"])
        if op in ("norm", "norm_bwd"):
            c = dict(op=op, T=_log(rng, 1, 40000), D=16 * _log(rng, 4, 512), dtype=rng.choice([BF16, BF16, FP32]), residual=rng.random() < 0.6)
            if op == "norm":
                c["out"] = rng.choice([c["dtype"], F8])
        elif op == "rope":
            d = rng.choice([64, 64, 96, 128, 128, 256])
            n = rng.choice([1, 2, 3])
            half = d // 2
            cut = sorted(rng.sample(range(1, half // 4), n - 1))  # sections of whole fours
            axes = [4 * (b - a) for a, b in zip([0] + cut, cut + [half // 4])]
            if rng.random() < 0.3 and axes[-1] > 4:  # the last dimensions do not turn
                axes[-1] -= 4
            c = dict(op=op, B=_log(rng, 1, 32), T=_log(rng, 1, 20000), heads=rng.choice([1, 3, 8, 24, 32]), d=d, axes=",".join(map(str, axes)),
                     layout=rng.choice(["pairs", "halves"]), shared=rng.random() < 0.5, far=_log(rng, 16, 2000000), dtype=rng.choice([BF16, BF16, FP32]), inverse=rng.random() < 0.4)
        else:
            T = _log(rng, 1, 64) if rng.random() < 0.4 and not op.endswith("bwd") else _log(rng, 1, 20000)
            c = dict(op=op, T=T, K=16 * _log(rng, 6, 512))
            c["N" if op.startswith("linear") else "F"] = 16 * _log(rng, 6, 768)
            c["dtype"] = BF16 if op.endswith("bwd") else rng.choice([BF16, BF16, F8])
            if op.startswith("linear"):
                c |= dict(bias=rng.random() < 0.6, act=rng.choice(["none", "relu", "gelu", "silu"]), residual=op == "linear" and rng.random() < 0.4)
            else:
                c["act"] = rng.choice(["silu", "silu", "gelu", "relu"])
        w = work(c)
        if w["flops"] < 1.6e12 and w["bytes"] < 5.2e8:
            return c


def _axes(c):
    return tuple(int(a) for a in c["axes"].split(","))


def work(c):
    op = c["op"]
    if op == "rope":
        n = c["B"] * c["T"] * c["heads"] * c["d"]
        return {"bytes": 2.0 * n * (2 if c["dtype"] == BF16 else 4) + 4.0 * c["B"] * c["T"] * len(_axes(c)), "flops": 3.0 * n}
    if op in ("norm", "norm_bwd"):
        n, e = c["T"] * c["D"], 2 if c["dtype"] == BF16 else 4
        if op == "norm":
            rows = n * e + (2 * n * e if c["residual"] else 0)  # x; r and h
            rows += n + 4 * c["T"] if c["out"] == F8 else n * e
            return {"bytes": float(rows + 4 * c["D"] + 4 * c["T"]), "flops": 5.0 * n}
        return {"bytes": float(n * e * (4 if c["residual"] else 3) + 4 * c["T"] + 8 * c["D"]), "flops": 8.0 * n}
    gated = op.startswith("gated")
    T, K, N = c["T"], c["K"], 2 * c["F"] if gated else c["N"]
    e = 1 if c["dtype"] == F8 else 2
    if not op.endswith("bwd"):
        out = T * (c["F"] if gated else N) * 2
        more = 4 * (T + N) if c["dtype"] == F8 else 0
        more += 0 if gated else (4 * N if c["bias"] else 0) + (2 * T * N if c["residual"] else 0)
        return {"bytes": float((T * K + N * K) * e + out + more), "flops": 2.0 * T * N * K}
    z = T * N * 2 if gated or c["act"] != "none" else 0
    dy = T * (c["F"] if gated else N) * 2
    db = 4 * N if not gated and c["bias"] else 0
    return {"bytes": float(2 * (T * K + N * K) * 2 + dy + z + db), "flops": 4.0 * T * N * K}


# ----------------------------------------------------------------------------- the inputs
def _rows8(x):
    """Rows of fp32 as e4m3 values and one power-of-two scale a row, none above 448."""
    m, e = torch.frexp(x.abs().amax(1))
    # the least power of two that brings the largest magnitude m 2^e to 448 = 0.875 * 2^9 or below
    e = e - 9 + (m > 0.875).to(e.dtype)
    scale = torch.ldexp(torch.ones_like(m), e.clamp(-126, 127))
    return (x / scale[:, None]).to(E4M3), scale


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    op, s = c["op"], {"c": c}
    if op == "rope":
        B, T, H, d, A = c["B"], c["T"], c["heads"], c["d"], len(_axes(c))
        # one of the three parts of a packed projection [B, T, 3, heads, d], in bf16 or fp32
        s["x"] = randn(B, T, 3, H, d).to(_DT[c["dtype"]])[:, :, 1]
        if T == 1:  # one token each of B sequences, up to `far` along
            pos = torch.randint(0, c["far"], (B, 1, A), generator=g, device="cuda")
        else:  # a grid of tokens in order, its inner sides alike, from an origin that the seed gives
            side = max(1, round(T ** (1.0 / A)))
            n = torch.arange(T, device="cuda")
            grid = [n // side ** (A - 1)] + [n // side ** (A - 1 - a) % side for a in range(1, A)]
            pos = torch.stack(grid, 1)[None] + torch.randint(0, c["far"], (B, 1, A), generator=g, device="cuda")
        s["pos"] = pos.to(torch.int32).contiguous()
        s["axes"] = _axes(c)
        return s
    if op in ("norm", "norm_bwd"):
        T, D, dt = c["T"], c["D"], _DT[c["dtype"]]
        chan = torch.exp(0.5 * randn(D))  # channels of unlike size, as residual streams have
        s["w"] = 1 + 0.1 * randn(D)
        x = (randn(T, D) * chan).to(dt)
        if op == "norm":
            s["x"] = x
            s["r"] = (randn(T, D) * chan).to(dt) if c["residual"] else None
        else:
            s["h"] = x
            s["rstd"] = (x.double().square().mean(1) + EPS).rsqrt().float()
            s["dy"] = (randn(T, D) / 16).to(dt)
            s["dh"] = (randn(T, D) / 16).to(dt) if c["residual"] else None
        return s
    gated = op.startswith("gated")
    T, K, N = c["T"], c["K"], 2 * c["F"] if gated else c["N"]
    x, W = randn(T, K) * torch.exp(0.25 * randn(K)), randn(N, K) / math.sqrt(K)
    if c["dtype"] == F8:
        s["x"], s["xs"] = _rows8(x)
        s["W"], s["ws"] = _rows8(W)
    else:
        s["x"], s["W"] = x.bfloat16(), W.bfloat16()
        s["xs"] = s["ws"] = None
    del x, W
    if not gated:
        s["b"] = 0.1 * randn(N) if c["bias"] else None
        s["r"] = randn(T, N).bfloat16() if c["residual"] else None
    if op.endswith("bwd"):
        s["dy"] = (randn(T, c["F"] if gated else N) / 16).bfloat16()
        s["z"] = randn(T, N).bfloat16() if gated or c["act"] != "none" else None
    return s


# ----------------------------------------------------------------------------- the plain forms
_C = math.sqrt(8 / math.pi)


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp(min=0)
    return z / (1 + torch.exp(-z if act == "silu" else -_C * (z + 0.044715 * z * z * z)))


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p + z * p * (1 - p)
    p = 1 / (1 + torch.exp(-_C * (z + 0.044715 * z * z * z)))
    return p + z * p * (1 - p) * _C * (1 + 3 * 0.044715 * z * z)


def _stands_for(q, scale):
    return q.bfloat16().mul_(scale[:, None])  # four bits times a power of two: exact


def _angles(s, c):
    """cos and sin of every token's pairs, [B, T, 1, pairs], angles in 64 bits."""
    axes, i = s["axes"], 0
    turn = []
    for a, n in enumerate(axes):
        k = torch.arange(n, device="cuda", dtype=torch.float64)
        theta = 10000.0 ** (-(k + i) / sum(axes) if c["shared"] else -k / n)
        turn.append(s["pos"][..., a:a + 1].double() * theta)
        i += n
    t = torch.cat(turn, -1)[:, :, None]
    return t.cos(), (-t if c["inverse"] else t).sin()


def _turn(x, cos, sin, layout, d):
    P = cos.shape[-1]
    if layout == "pairs":
        a, b = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        return torch.cat((y, x[..., 2 * P:]), -1)
    a, b = x[..., :P], x[..., P:2 * P]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, x[..., 2 * P:]), -1)


def _plain(s, c):
    op = c["op"]
    if op == "rope":
        cos, sin = _angles(s, c)
        y = _turn(s["x"].float(), cos.float(), sin.float(), c["layout"], c["d"])
        return y.to(s["x"].dtype).transpose(1, 2).contiguous()
    if op == "norm":
        h = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)
        v = h.float()
        rstd = (v.square().mean(1) + EPS).rsqrt()
        y = v * rstd[:, None] * s["w"]
        y = _stands_for(*_rows8(y)) if c["out"] == F8 else y.to(h.dtype)
        return (y, h, rstd) if c["residual"] else (y, rstd)
    if op == "norm_bwd":
        xh = s["h"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["w"]
        dx = s["rstd"][:, None] * (g - xh * (g * xh).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return dx.to(s["h"].dtype), (dy * xh).sum(0)
    if op.endswith("bwd"):
        dy = s["dy"].float()
        if op == "gated_bwd":
            g, u = s["z"].float().chunk(2, 1)
            dz = torch.cat((dy * u * _act_slope(g, c["act"]), dy * _act(g, c["act"])), 1)
        else:
            dz = dy if s["z"] is None else dy * _act_slope(s["z"].float(), c["act"])
        out = ((dz @ s["W"].float()).bfloat16(), (dz.T @ s["x"].float()).bfloat16())
        return out + (dz.sum(0),) if c.get("bias") else out
    z = s["x"].float() @ s["W"].float().T
    if s["xs"] is not None:
        z = z * s["xs"][:, None] * s["ws"]
    if op == "gated":
        g, u = z.chunk(2, 1)
        return (_act(g, c["act"]) * u).bfloat16()
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, c["act"])
    return (y if s["r"] is None else y + s["r"].float()).bfloat16()


def run(s):
    c = s["c"]
    if not own:
        return _plain(s, c)
    import paper_2605_15684_gb300 as gb

    op = c["op"]
    act = None if c.get("act") == "none" else c.get("act")
    if op == "rope":
        B, T, H, d = s["x"].shape
        y = torch.empty((B, H, T, d), dtype=s["x"].dtype, device="cuda")
        gb.rope_axes(s["x"], s["pos"], s["axes"], layout=c["layout"], shared=c["shared"], inverse=c["inverse"], out=y.transpose(1, 2))
        return y
    if op == "norm":
        if c["out"] == F8:
            q, scale, h, rstd = gb.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS, e4m3=True)
            y = _stands_for(q, scale)
        else:
            y, h, rstd = gb.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS)
        return (y, h, rstd) if c["residual"] else (y, rstd)
    if op == "norm_bwd":
        return gb.rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"])
    if op == "linear":
        return gb.linear(s["x"], s["W"], bias=s["b"], residual=s["r"], act=act, x_scale=s["xs"], w_scale=s["ws"])
    if op == "linear_bwd":
        dx, dW, db = gb.linear_backward(s["dy"], s["x"], s["W"], z=s["z"], act=act, bias=c["bias"])
        return (dx, dW, db) if c["bias"] else (dx, dW)
    if op == "gated":
        return gb.gated_linear(s["x"], s["W"], act=act, x_scale=s["xs"], w_scale=s["ws"])
    return gb.gated_linear_backward(s["dy"], s["x"], s["W"], s["z"], act=act)


# ----------------------------------------------------------------------------- the definitions, in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    up = lambda n: None if s.get(n) is None else s[n].double()  # noqa: E731
    op = c["op"]
    sig = torch.special.expit
    inner = lambda z: z if c["act"] == "silu" else (2 / math.pi) ** 0.5 * 2 * (z + 0.044715 * z ** 3)  # noqa: E731
    f = {"none": lambda z: z, "relu": torch.relu}.get(c.get("act"), lambda z: z * sig(inner(z)))
    if op == "rope":
        # as a product of complex numbers, pair by pair
        P, x = sum(s["axes"]), up("x")
        which = torch.repeat_interleave(torch.arange(len(s["axes"])), torch.tensor(s["axes"])).cuda()
        rank = torch.cat([torch.arange(n) for n in s["axes"]]).cuda().double()
        of = torch.cat([torch.full((n,), n) for n in s["axes"]]).cuda().double()
        power = torch.arange(P, device="cuda").double() / P if c["shared"] else rank / of
        ang = s["pos"].double()[..., which] * torch.exp(-power * math.log(10000.0))
        z = torch.polar(torch.ones_like(ang), ang)[:, :, None]
        z = z.conj() if c["inverse"] else z
        re, im = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if c["layout"] == "pairs" else (x[..., :P], x[..., P:2 * P])
        w = torch.complex(re.contiguous(), im.contiguous()) * z
        y = x.clone()
        if c["layout"] == "pairs":
            y[..., 0:2 * P:2], y[..., 1:2 * P:2] = w.real, w.imag
        else:
            y[..., :P], y[..., P:2 * P] = w.real, w.imag
        return y.transpose(1, 2).contiguous()
    if op == "norm":
        h = s["x"] if s["r"] is None else (up("x") + up("r")).to(s["x"].dtype)
        hd = h.double()
        n = torch.linalg.vector_norm(hd, dim=1)
        rstd = 1 / torch.sqrt(n * n / c["D"] + EPS)
        y = torch.einsum("td,t,d->td", hd, rstd, up("w"))
        if c["out"] == F8:
            scale = 2.0 ** torch.ceil(torch.log2(y.abs().amax(1, keepdim=True) / 448))
            y = (y / scale).to(E4M3).double() * scale
        return (y, hd, rstd) if c["residual"] else (y, rstd)
    if op == "norm_bwd":
        h, w, k, dy = up("h"), up("w"), up("rstd"), up("dy")
        along = torch.einsum("td,d,td->t", dy, w, h) * k ** 3 / c["D"]
        dx = torch.einsum("td,d,t->td", dy, w, k) - h * along[:, None]
        return dx if s["dh"] is None else dx + up("dh"), torch.einsum("td,td,t->d", dy, h, k)
    if op.endswith("bwd"):
        dy, z = up("dy"), up("z")
        if z is not None:
            z.requires_grad_(True)
            F = z.shape[1] // 2
            y = f(z[:, :F]) * z[:, F:] if op == "gated_bwd" else f(z)
            (dz,) = torch.autograd.grad(y, z, dy)
        else:
            dz = dy
        out = (torch.einsum("tn,nk->tk", dz, up("W")), torch.einsum("tn,tk->nk", dz, up("x")))
        return out + (torch.einsum("tn->n", dz),) if c.get("bias") else out
    x, W = up("x"), up("W")
    if s["xs"] is not None:
        x, W = x * up("xs")[:, None], W * up("ws")[:, None]
    if op == "gated":
        F = c["F"]
        return f(torch.einsum("tk,nk->tn", x, W[:F])) * torch.einsum("tk,nk->tn", x, W[F:])
    z = torch.einsum("tk,nk->tn", x, W)
    z = z if s["b"] is None else z + up("b")
    return f(z) if s["r"] is None else f(z) + up("r")
