"""GPU tests of a layer's operators at their edges: values and layouts that are allowed and seldom met."""
import pytest
import torch

import paper_2605_15684_gb300 as gb
from paper_2605_15684_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


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
