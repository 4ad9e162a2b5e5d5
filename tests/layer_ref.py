"""Plain 64-bit forms of a layer's operators, and how far a kernel may be from them.

Tolerances count roundings. A 16-bit result is off by 2^-8 of its value (half a step of bf16). A sum of n products in fp32
is taken as off by n 2^-23 of the sum of their magnitudes (a rounding of 2^-24 and an alignment of as much a term).
An activation's fp32 form is taken as off by 2^-16 of its value (the exponential and the quotient, some 2^-20 each, and
2^-24 |t| of the argument t <= 90, past which the value is 0 or z), and it stretches an error of z by 1.2 at most.
"""
import math

import torch

C = 2 * math.sqrt(2 / math.pi)
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def half_step(t):
    return torch.finfo(t).eps / 2


def act(z, name):
    if name is None:
        return z
    if name == "relu":
        return torch.relu(z)  # its slope at 0 is 0
    return z * torch.sigmoid(z if name == "silu" else C * (z + 0.044715 * z ** 3))


def e4m3_rows(x):
    """e4m3 rows and their power-of-two scales of a 2-D tensor."""
    a = x.double().abs().amax(1, keepdim=True)
    s = torch.where(a > 0, torch.exp2(torch.ceil(torch.log2(a / 448).clamp(min=-126))), torch.ones_like(a))
    return (x.double() / s).float().to(E4M3), s[:, 0].float()


def operand(x, scale):
    return x.double() if scale is None else x.double() * scale.double()[:, None]


def linear(x, W, bias=None, residual=None, name=None, xs=None, ws=None):
    """(y, z, tolerance of y, tolerance of z before its rounding)"""
    a, b = operand(x, xs), operand(W, ws)
    z = a @ b.T
    ez = (a.abs() @ b.abs().T) * (x.shape[1] * 2.0 ** -23)
    if bias is not None:
        z = z + bias.double()
        ez = ez + 2.0 ** -23 * z.abs()
    y = act(z, name)
    ey = 1.2 * ez + 2.0 ** -16 * y.abs()
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2.0 ** -23 * y.abs()
    return y, z, ey + (y.abs() + ey) * 2.0 ** -8 + 1e-30, ez


def gated(x, W, name, xs=None, ws=None):
    _, z, _, ez = linear(x, W, xs=xs, ws=ws)
    F = z.shape[1] // 2
    g, u, eg, eu = z[:, :F], z[:, F:], ez[:, :F], ez[:, F:]
    h = act(g, name)
    eh = 1.2 * eg + 2.0 ** -16 * h.abs()
    y = h * u
    ey = eh * u.abs() + h.abs() * eu + eh * eu
    return y, z, ey + (y.abs() + ey) * 2.0 ** -8 + 1e-30, ez


def slope(z, name, is_gated, dy):
    """dz of z's gradient by autograd in 64 bits."""
    z = z.double().requires_grad_(True)
    F = z.shape[1] // 2
    y = act(z[:, :F], name) * z[:, F:] if is_gated else act(z, name)
    return torch.autograd.grad(y, z, dy.double())[0]


def linear_backward(dy, x, W, z, name, is_gated=False):
    """((dx, tolerance), (dW, tolerance), (db, tolerance))"""
    dz = dy.double() if name is None else slope(z, name, is_gated, dy)
    # with an activation dz is rounded to bf16; its fp32 form is off by 2^-14 of |dy| (|u|): the slope's terms are
    # up to 1.2 and cancel
    up = dy.double().abs()
    if is_gated:
        up = torch.cat((up * z.double()[:, z.shape[1] // 2:].abs(), up * act(z.double()[:, :z.shape[1] // 2], name).abs()), 1)
    e = torch.zeros_like(dz) if name is None else dz.abs() * 2.0 ** -8 + up * 2.0 ** -14
    out = []
    for r, m, n in ((dz @ W.double(), e @ W.double().abs() + (dz.abs() @ W.double().abs()) * (dz.shape[1] * 2.0 ** -23), None),
                    (dz.T @ x.double(), e.T @ x.double().abs() + (dz.T.abs() @ x.double().abs()) * (dz.shape[0] * 2.0 ** -23), None)):
        out.append((r, m + (r.abs() + m) * 2.0 ** -8 + 1e-30))
    db = dz.sum(0)
    ez = torch.zeros_like(dz) if name is None else up * 2.0 ** -14
    out.append((db, ez.sum(0) + dz.abs().sum(0) * (dz.shape[0] * 2.0 ** -23) + 1e-30))
    return out


def norm(h, w, eps):
    h = h.double()
    rstd = (h.square().mean(1) + eps).rsqrt()
    return h * rstd[:, None] * w.double(), rstd


def norm_backward(dy, h, w, rstd, dh):
    """By autograd in 64 bits (rstd follows from h and eps; the given one stands for both)."""
    h = h.double().requires_grad_(True)
    w = w.double().requires_grad_(True)
    eps = (rstd.double() ** -2 - h.detach().square().mean(1)).clamp(min=0)
    y = h * (h.square().mean(1) + eps).rsqrt()[:, None] * w
    dx, dw = torch.autograd.grad(y, (h, w), dy.double())
    return (dx if dh is None else dx + dh.double()), dw


def rope(x, pos, axes, base=10000.0, layout="pairs", shared=False, inverse=False):
    """x [B, T, heads, d]"""
    x, P, j = x.double(), sum(axes), 0
    pos = pos if pos.dim() == 3 else pos[None].expand(x.shape[0], -1, -1)
    ang = []
    for a, n in enumerate(axes):
        i = torch.arange(n, dtype=torch.float64, device=x.device)
        ang.append(pos[..., a:a + 1].double() * base ** (-((i + j) / P if shared else i / n)))
        j += n
    ang = torch.cat(ang, -1)[:, :, None] * (-1 if inverse else 1)
    c, s = ang.cos(), ang.sin()
    y = x.clone()
    u, v = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "pairs" else (slice(0, P), slice(P, 2 * P))
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., u] * s + x[..., v] * c
    return y


def near(got, want, tol, what=""):
    err = (got.double() - want).abs()
    assert got.shape == want.shape
    assert bool((err <= tol).all()), f"{what}: off by {float((err - tol).max()):.3e} more than {float(tol.flatten()[(err - tol).argmax()]):.3e}"
