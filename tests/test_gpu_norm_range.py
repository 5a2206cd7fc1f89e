"""Gradients whose norm passes fp32's range: the update goes by the norm that the
caller sees.  Powers of two, so that every expected value is exact."""
import math

import pytest
import torch

from paper_2508_06993_amd.runtime import Parameters

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 127


@pytest.mark.parametrize("count", [4, 1 << 16], ids=["one-launch", "two-launches"])
def test_update_of_a_norm_past_fp32(gpu, count):
    """2^127 sqrt(4) = 2^128 is no fp32 value: the norm is infinite, the step left out."""
    g, p, m, v, ema = (torch.full((count,), x, device="cuda") for x in (0.0, 1.0, 0.5, 0.25, 2.0))
    g[:4] = BIG
    lst = Parameters([g], [p], [m], [v], ema=[ema])
    assert math.isinf(float(lst.adamw(0.1, max_norm=1.0))) and int(lst.step) == 0
    for x, want in ((p, 1.0), (m, 0.5), (v, 0.25), (ema, 2.0)):
        assert bool((x == want).all())
    # with a scale that brings the norm back it is made
    assert float(lst.adamw(0.1, max_norm=1.0, scale=2.0 ** -8)) == 2.0 ** 120
    assert int(lst.step) == 1 and not bool((p == 1.0).any())
    # just inside: 2^127 sqrt(3)
    g[3] = 0
    assert math.isfinite(float(lst.adamw(0.1, max_norm=1.0))) and int(lst.step) == 2


@pytest.mark.parametrize("count", [4, 1 << 16], ids=["one-launch", "two-launches"])
def test_clip_of_a_norm_past_fp32(gpu, count):
    """The gradients are finite, and so are their clipped copies: 2^127 / 2^128."""
    g, out = torch.zeros(count, device="cuda"), torch.ones(count, device="cuda")
    g[:4] = BIG
    assert math.isinf(float(Parameters([g], clipped=[out]).clip(1.0)))
    assert bool((out[:4] == 0.5).all()) and not bool(out[4:].any())


def test_update_of_a_large_list(gpu):
    """Past the size from which the arrays are streamed."""
    n = 9_000_000
    g, p, m, v = (torch.full((n,), x, device="cuda") for x in (0.0, 1.0, 0.5, 0.25))
    g[5::n // 4] = BIG
    lst = Parameters([g], [p], [m], [v])
    assert math.isinf(float(lst.adamw(0.1, max_norm=1.0))) and int(lst.step) == 0
    assert bool((p == 1).all()) and bool((m == 0.5).all()) and bool((v == 0.25).all())
