"""Refusals of a layer's operators: every bad call is an error on the host, before any device work."""
import ctypes

import pytest
import torch

from paper_2605_15684_gb300 import api, build, layer

FAKE = 0x100000  # a 16-byte aligned, never dereferenced address
ODD = FAKE + 4


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load_library()


def linear_desc(**kw):
    d = dict(T=4, N=64, K=64, dtype=api.SSBA_BF16, act=0, gated=0)
    d.update(kw)
    return ctypes.byref(layer._LinearDesc(**d))


def rope_desc(**kw):
    d = dict(B=1, T=4, heads=2, head_dim=64, axes=2, sections=(16, 16, 0, 0), layout=0, shared=0, inverse=0,
             dtype=api.SSBA_BF16, base=10000.0)
    d.update(kw)
    d["sections"] = (ctypes.c_int32 * 4)(*d["sections"])
    return ctypes.byref(layer._RopeDesc(**d))


def S(*v):
    return (ctypes.c_int64 * 3)(*v)


INV, UNS, WS = api.SSBA_ERR_INVALID, api.SSBA_ERR_UNSUPPORTED, api.SSBA_ERR_WORKSPACE


@pytest.mark.parametrize("args,code", [
    (dict(T=-1), INV), (dict(D=0), INV), (dict(dtype=2), INV), (dict(dtype=7), INV), (dict(D=60), UNS), (dict(D=16392), UNS),
    (dict(eps=-1.0), INV), (dict(eps=float("inf")), INV), (dict(eps=float("nan")), INV), (dict(r=FAKE), INV), (dict(h=FAKE), INV),
    (dict(x=None), INV), (dict(w=None), INV), (dict(y=None), INV), (dict(rstd=None), INV), (dict(x=ODD), INV), (dict(w=ODD), INV),
    (dict(y=ODD), INV), (dict(scale=FAKE + 2), INV),
])
def test_norm_refusals(lib, args, code):
    a = dict(x=FAKE, r=None, w=FAKE, T=4, D=64, dtype=0, eps=1e-6, h=None, y=FAKE, scale=None, rstd=FAKE)
    a.update(args)
    assert lib.ssba_rms_norm(*a.values(), None) == code
    assert b"ssba_rms_norm" in lib.ssba_last_error()


@pytest.mark.parametrize("args,code", [
    (dict(T=-1), INV), (dict(D=60), UNS), (dict(dtype=2), INV), (dict(dy=None), INV), (dict(h=None), INV), (dict(w=None), INV),
    (dict(rstd=None), INV), (dict(dx=None), INV), (dict(dw=None), INV), (dict(dh=ODD), INV), (dict(ws=None), WS), (dict(n=16), WS),
    (dict(ws=ODD), WS),
])
def test_norm_backward_refusals(lib, args, code):
    a = dict(dy=FAKE, h=FAKE, w=FAKE, rstd=FAKE, dh=None, T=400, D=64, dtype=0, dx=FAKE, dw=FAKE, ws=FAKE, n=1 << 30)
    a.update(args)
    assert lib.ssba_rms_norm_backward(*a.values(), None) == code


@pytest.mark.parametrize("desc,args,code", [
    (dict(T=-1), {}, INV), (dict(N=0), {}, INV), (dict(K=0), {}, INV), (dict(dtype=1), {}, INV), (dict(dtype=3), {}, INV), (dict(act=4), {}, INV),
    (dict(act=-1), {}, INV), (dict(gated=1), {}, INV), (dict(N=60), {}, UNS), (dict(K=60), {}, UNS), (dict(N=1 << 18), {}, UNS),
    (dict(K=1 << 18), {}, UNS), (dict(T=(1 << 24) + 1), {}, UNS),
    (dict(dtype=2, K=72), dict(xs=FAKE, ws=FAKE), UNS), (dict(dtype=2), {}, INV), (dict(dtype=2), dict(xs=FAKE), INV), ({}, dict(ws=FAKE), INV),
    (dict(gated=1, act=3), dict(bias=FAKE), INV), (dict(gated=1, act=3), dict(r=FAKE), INV),
    ({}, dict(x=None), INV), ({}, dict(W=None), INV), ({}, dict(y=None), INV), ({}, dict(x=ODD), INV), ({}, dict(z=ODD), INV), ({}, dict(bias=ODD), INV),
])
def test_linear_refusals(lib, desc, args, code):
    a = dict(x=FAKE, W=FAKE, xs=None, ws=None, bias=None, r=None, y=FAKE, z=None)
    a.update(args)
    assert lib.ssba_linear(linear_desc(**desc), *a.values(), None) == code


@pytest.mark.parametrize("desc,args,code", [
    (dict(dtype=2), {}, INV), (dict(N=60), {}, UNS), (dict(gated=1, act=3), dict(db=FAKE), INV), ({}, dict(W=None), INV), ({}, dict(x=None), INV),
    ({}, dict(dy=None), INV), (dict(act=2), {}, INV), (dict(act=2), dict(z=FAKE, ws=None), WS), (dict(act=2), dict(z=FAKE, n=16), WS),
    ({}, dict(dx=ODD), INV), ({}, dict(db=FAKE + 2), INV),
])
def test_linear_backward_refusals(lib, desc, args, code):
    a = dict(dy=FAKE, x=FAKE, W=FAKE, z=None, dx=FAKE, dW=FAKE, db=None, ws=FAKE, n=1 << 30)
    a.update(args)
    assert lib.ssba_linear_backward(linear_desc(**desc), *a.values(), None) == code
    assert lib.ssba_linear_backward(None, *a.values(), None) == INV


@pytest.mark.parametrize("desc,args,code", [
    (dict(B=-1), {}, INV), (dict(T=-1), {}, INV), (dict(heads=0), {}, INV), (dict(head_dim=0), {}, INV), (dict(axes=0), {}, INV), (dict(axes=5), {}, INV),
    (dict(sections=(16, 0, 0, 0)), {}, INV), (dict(sections=(16, 17, 0, 0)), {}, INV), (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 0, 0)), {}, INV),
    (dict(layout=2), {}, INV), (dict(base=1.0), {}, INV), (dict(base=float("nan")), {}, INV), (dict(base=float("inf")), {}, INV), (dict(dtype=2), {}, INV),
    (dict(head_dim=65), {}, UNS), (dict(head_dim=258), {}, UNS), (dict(B=1 << 20, T=1 << 20), {}, UNS),
    ({}, dict(x=None), INV), ({}, dict(pos=None), INV), ({}, dict(out=None), INV), ({}, dict(xs=None), INV), ({}, dict(os=S(0, -64, 64)), INV),
    ({}, dict(x=FAKE + 2), INV), (dict(layout=1), dict(x=FAKE + 1), INV), ({}, dict(xs=S(0, 65, 64)), INV), ({}, dict(pos=FAKE + 2), INV), ({}, dict(pb=-1), INV),
])
def test_rope_refusals(lib, desc, args, code):
    a = dict(x=FAKE, xs=S(512, 128, 64), pos=FAKE, pb=0, out=FAKE, os=S(512, 128, 64))
    a.update(args)
    assert lib.ssba_rope_axes(rope_desc(**desc), *a.values(), None) == code


def test_no_rows_is_no_work(lib):
    assert lib.ssba_rms_norm(None, None, None, 0, 64, 0, 1e-6, None, None, None, None, None) == api.SSBA_OK
    assert lib.ssba_linear(linear_desc(T=0), *[None] * 8, None) == api.SSBA_OK
    assert lib.ssba_rope_axes(rope_desc(T=0), None, S(0, 0, 0), None, 0, None, S(0, 0, 0), None) == api.SSBA_OK


def test_workspace_sizes(lib):
    assert lib.ssba_linear_backward_workspace_bytes(linear_desc(T=100, N=64, act=2)) >= 100 * 64 * 2 + 64 * 4
    assert lib.ssba_linear_backward_workspace_bytes(linear_desc(T=100, N=64, act=3, gated=1)) == 100 * 128 * 2
    assert lib.ssba_linear_backward_workspace_bytes(linear_desc(N=60)) == 0
    assert lib.ssba_rms_norm_backward_workspace_bytes(100, 64, 0) >= 64 * 4
    assert lib.ssba_rms_norm_backward_workspace_bytes(100, 63, 0) == 0


def test_python_refuses_what_is_not_on_the_gpu(lib):
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    for call in (lambda: layer.rms_norm(x, w), lambda: layer.rms_norm_backward(x, x, w, w[:4]), lambda: layer.linear(x, x),
                 lambda: layer.gated_linear(x, x), lambda: layer.linear_backward(x, x, x), lambda: layer.rms_norm(w, w),
                 lambda: layer.gated_linear_backward(x, x, x, x), lambda: layer.rms_norm(x.half(), w), lambda: layer.linear(None, x),
                 lambda: layer.rope_axes(x.view(1, 2, 2, 64), torch.zeros(2, 2, dtype=torch.int32), (16, 16)),
                 lambda: layer.rope_axes(x, None, (16,))):
        with pytest.raises(api.SsbaError):
            call()


def test_rope_descriptor_refusals():
    ok = (1, 4, 2, 64, (16, 16), "pairs", False, False, torch.bfloat16, 10000.0)
    layer._rope_desc(ok)
    for i, v in ((4, ()), (4, (1,) * 5), (4, (16, 0)), (4, (2 ** 33, 1)), (5, "interleaved"), (1, 2 ** 31)):
        with pytest.raises(api.SsbaError):
            layer._rope_desc((*ok[:i], v, *ok[i + 1:]))


@pytest.mark.parametrize("shape,strides,dense", [
    ((2, 3, 4, 64), (768, 256, 64, 1), True), ((2, 3, 4, 64), (768, 64, 192, 1), True), ((2, 3, 4, 64), (0, 256, 64, 1), False),
    ((1, 3, 4, 64), (0, 256, 64, 1), True), ((2, 3, 4, 64), (768, 256, 32, 1), False), ((1, 3, 1, 64), (0, 63, 7, 1), False),
])
def test_overlapping_outputs_are_seen(shape, strides, dense):
    assert layer._dense_heads(shape, strides) is dense


def test_outputs_on_other_tensors_are_refused(lib):
    """Addresses far apart, but for one output that overlaps one other tensor of its call."""
    at = [0x100000000 * (i + 1) for i in range(12)]
    x, r, w, h, y, sc, k = at[:7]
    norm = lambda **a: lib.ssba_rms_norm(*{**dict(x=x, r=r, w=w, T=4, D=64, dtype=0, eps=1e-6, h=h, y=y, s=sc, k=k), **a}.values(), None)  # noqa: E731
    for bad in (dict(h=x + 16), dict(h=w), dict(y=x), dict(y=h + 16), dict(y=r), dict(k=y + 4), dict(s=h), dict(s=k), dict(s=None, y=x + 16)):
        assert norm(**bad) == INV, bad
        assert b"lies on" in lib.ssba_last_error()
    dy, hh, dh, dx, dw, ws = at[:6]
    back = lambda **a: lib.ssba_rms_norm_backward(*{**dict(dy=dy, h=hh, w=at[6], k=at[7], dh=dh, T=400, D=64, dtype=0, dx=dx, dw=dw, ws=ws, n=1 << 28), **a}.values(), None)  # noqa: E731
    for bad in (dict(dx=hh), dict(dx=dy + 16), dict(dw=dx), dict(ws=hh), dict(dx=ws)):
        assert back(**bad) == INV, bad
    X, W, xs, wsc, b, res, Y, Z = at[:8]
    lin = lambda d, **a: lib.ssba_linear(linear_desc(**d), *{**dict(x=X, W=W, xs=None, ws=None, b=b, r=res, y=Y, z=Z), **a}.values(), None)  # noqa: E731
    for bad in (dict(y=X), dict(y=W + 16), dict(y=res + 16), dict(z=Y), dict(z=res), dict(y=b), dict(z=X)):
        assert lin({}, **bad) == INV, bad
    assert lin(dict(gated=1, act=3), b=None, r=None, z=Y + 4 * 64 * 2 - 16) == INV
    bwd = lambda **a: lib.ssba_linear_backward(linear_desc(act=2), *{**dict(dy=at[0], x=at[1], W=at[2], z=at[3], dx=at[4], dW=at[5], db=at[6], ws=at[7], n=1 << 28), **a}.values(), None)  # noqa: E731
    for bad in (dict(dx=at[0]), dict(dx=at[1]), dict(dW=at[2]), dict(dW=at[4] + 16), dict(db=at[3]), dict(ws=at[0]), dict(ws=at[5]), dict(dx=at[7])):
        assert bwd(**bad) == INV, bad


@pytest.mark.parametrize("apart,xs,os", [
    (64, (768, 192, 64), (768, 192, 64)),     # a head further on in the same tensor
    (2, (768, 192, 64), (768, 192, 64)),      # two dimensions further on
    (192 * 3, (768, 192, 64), (768, 192, 64)),
    (0, (768, 192, 64), (768, 64, 256)),      # the same tensor in another order
    (1536, (768, 192, 64), (1536, 192, 64)),
])
def test_rope_refuses_an_output_on_its_input(lib, apart, xs, os):
    x = 0x100000000
    rc = lib.ssba_rope_axes(rope_desc(B=4, heads=3), x, S(*xs), 0x900000000, 0, x + 2 * apart, S(*os), None)
    assert rc == INV and b"lies on" in lib.ssba_last_error()


@pytest.mark.parametrize("pb,at", [(0, -4 * 2 * 4 + 4), (0, 0), (0, 4 * (768 * 3 + 192 * 3 + 64 * 2 + 64) - 4), (8, -4 * (3 * 8 + 4 * 2) + 4), (8, -4 * 3 * 8)])
def test_rope_refuses_an_output_on_its_positions(lib, pb, at):
    out = 0x100000000
    rc = lib.ssba_rope_axes(rope_desc(B=4, heads=3, dtype=api.SSBA_FP32), 0x900000000, S(768, 192, 64), out + at, pb, out, S(768, 192, 64), None)
    assert rc == INV and b"lies on pos" in lib.ssba_last_error()


def test_timeout_hook_refusals(lib):
    for d in (dict(T=0), dict(dtype=2), dict(N=60)):
        assert lib.ssba_test_linear_timeout(linear_desc(**d), FAKE, FAKE, FAKE, 1000000, None) in (INV, UNS)
    assert lib.ssba_test_linear_timeout(None, FAKE, FAKE, FAKE, 1000000, None) == INV
