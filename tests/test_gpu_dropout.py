"""Dropout on the GPU against the generator's definition: which elements are kept
is exact; a kept value has the error of fp32 arithmetic (the factor's rounding, the
product's, the sum's: 2^-24 of their magnitudes each) and of the last rounding."""
import numpy as np
import pytest
import torch

import cells4
import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import Dropout

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def spaced(x, pad, fill=7.0):
    wide = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]], wide


def kept_mask(rows, cols, rate, seed, index):
    draws = cells4.draws(range(rows * cols), seed, index)
    return torch.from_numpy((draws >= cells4.threshold(rate)).reshape(rows, cols))


def check(out, x, mask, rate, add, dtype):
    """out against 64 bits, element by element."""
    t = cells4.threshold(rate)
    x = x.double().cpu()
    y = torch.where(mask, x * (2.0 ** 32 / (2 ** 32 - t) if t < 2 ** 32 else 0.0), 0.0)
    mags = y.abs()
    if add is not None:
        y, mags = y + add.double().cpu(), mags + add.double().cpu().abs()
    bound = (3 * 2.0 ** -24 * mags + torch.finfo(TYPES[dtype]).eps / 2 * y.abs() * 1.001 +
             {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[dtype])
    err = (out.double().cpu() - y).abs()
    assert (err <= bound).all(), (err / bound).max()
    if add is None:
        assert (out.cpu()[~mask] == 0).all()


CASES = [  # rows, cols, spacings of x, gate, add and out
    (1, 1, (0, 0, 0, 0)), (1, 7, (0, 0, 0, 0)), (3, 5, (0, 0, 0, 0)), (4, 64, (0, 0, 0, 0)),
    (33, 8, (0, 0, 0, 0)), (16, 64, (8, 0, 16, 8)), (21, 100, (4, 4, 4, 4)),
    (17, 33, (1, 2, 3, 4)), (50, 16, (0, 1, 0, 0)), (9, 517, (0, 3, 0, 3)), (700, 3, (0, 0, 0, 1)),
    (2, 4100, (0, 0, 4, 0))]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pads", CASES)
def test_dropout(gpu, rows, cols, pads, dtype):
    rng = np.random.default_rng(rows * cols)
    new = lambda pad: spaced(torch.from_numpy(rng.standard_normal((rows, cols)))
                             .to(gpu, TYPES[dtype]), pad)
    (x, _), (gate, _), (add, _), (out, wide) = (new(p) for p in pads)
    for rate, use_gate, use_add in ((0.5, False, False), (0.1, True, False), (0.3, False, True),
                                    (0.0, True, True), (1.0, False, True), (0.9, True, True)):
        seed, index = int(rng.integers(2 ** 63)), int(rng.integers(2 ** 40))
        mask = kept_mask(rows, cols, rate, seed, index)
        if use_gate:
            mask &= gate.cpu() > 0
        out.fill_(3.0)
        got = Dropout(rate, seed)(x, out, gate=gate if use_gate else None,
                                  add=add if use_add else None, index=index)
        assert got is out
        check(out, x, mask, rate, add if use_add else None, dtype)
        assert (wide[:, cols:] == 7).all()


def test_far_elements(gpu):
    """The draws of elements past 2^32 draw on the counter's second word."""
    rows, cols = 70000, 65536
    x = torch.ones((rows, cols), dtype=torch.float16, device=gpu)
    Dropout(0.25, 99)(x, x, index=5)
    for first in (0, 2 ** 32 - 8, 2 ** 32, 2 ** 32 + 123456, rows * cols - 40):
        draws = cells4.draws(range(first, first + 40), 99, 5)
        got = x.reshape(-1)[first:first + 40].cpu().numpy() != 0
        assert np.array_equal(got, draws >= cells4.threshold(0.25))


def test_many_elements(gpu):
    """The share of kept elements, and no pattern from call to call: 5 sigma."""
    n = 1 << 22
    x = torch.ones(1, n, device=gpu)
    a, b = (Dropout(0.3, 1)(x, torch.zeros_like(x), index=k) != 0 for k in (0, 1))
    for p, hits in ((0.7, a), (0.7, b), (0.49, a & b)):
        assert abs(hits.sum().item() - n * p) < 5 * (n * p * (1 - p)) ** 0.5


@pytest.mark.parametrize("which", ["x", "gate", "add"])
@pytest.mark.parametrize("cols,pad", [(64, 0), (33, 5)])
def test_in_place(gpu, which, cols, pad):
    t = {k: spaced(torch.randn(40, cols, device=gpu), pad)[0] for k in ("x", "gate", "add")}
    drop = Dropout(0.4, 11)
    want = drop(t["x"], torch.zeros(40, cols, device=gpu), gate=t["gate"], add=t["add"], index=2)
    drop(t["x"], t[which], gate=t["gate"], add=t["add"], index=2)
    assert torch.equal(t[which], want)


def test_what_is_dropped_does_not_matter(gpu):
    x = torch.randn(64, 48, device=gpu)
    mask = kept_mask(64, 48, 0.5, 7, 0).to(gpu)
    dirty = torch.where(mask, x, torch.tensor(float("nan"), device=gpu))
    assert torch.equal(Dropout(0.5, 7)(dirty, torch.zeros_like(x)),
                       Dropout(0.5, 7)(x, torch.zeros_like(x)))
    # a gate of NaN is not positive; kept values that are not finite stay so
    gate = torch.ones_like(x)
    gate[0] = float("nan")
    x[1], x[2] = float("inf"), float("nan")
    out = Dropout(0.0, 7)(x, torch.zeros_like(x), gate=gate)
    assert (out[0] == 0).all() and torch.isinf(out[1]).all() and torch.isnan(out[2]).all()
    assert torch.equal(out[3:], x[3:])


def test_gradient(gpu):
    """ReLU and dropout, and their gradient, by differences in 64 bits of the
    function that the same call computes."""
    drop = Dropout(0.35, 1234)
    x = torch.randn(30, 50, device=gpu)
    x[x.abs() < 0.05] = 0.5          # no kink within a step
    g = torch.randn(30, 50, device=gpu)
    grad = drop(g, torch.zeros_like(x), gate=x, index=9)
    f = lambda v: drop(v, torch.zeros_like(x), gate=v, index=9).double()
    step = 2.0 ** -6
    quotient = (f(x + step) - f(x - step)) / (2 * step)
    # a value of at most 8 and its factor are rounded to 2^-24 of it: four times, over the step
    bound = 4 * 2.0 ** -24 * 8 * 2 / (2 * step)
    assert ((quotient - grad.double() / g.double()).abs() <= bound + 2.0 ** -22).all()


def test_shapes_and_device_step(gpu):
    """More dimensions are taken as rows of the last; the step on the device adds
    to the index, modulo 2^64."""
    x = torch.randn(3, 5, 8, 4, device=gpu)
    out = Dropout(0.5, 3)(x, torch.zeros_like(x), index=7)
    assert torch.equal(out.reshape(120, 4),
                       Dropout(0.5, 3)(x.reshape(120, 4), torch.zeros(120, 4, device=gpu), index=7))
    step = torch.tensor([5], device=gpu)
    assert torch.equal(Dropout(0.5, 3, step)(x, torch.zeros_like(x), index=2), out)
    step.fill_(-1)
    assert torch.equal(Dropout(0.5, 3, step)(x, torch.zeros_like(x), index=8), out)


def test_refusals(gpu):
    x = torch.zeros(10, 20, device=gpu)
    drop = Dropout(0.5, 1)
    for bad in (dict(out=torch.zeros(10, 21, device=gpu)),
                dict(out=torch.zeros(10, 20, device=gpu, dtype=torch.float16)),
                dict(out=torch.zeros(10, 20)), dict(gate=torch.zeros(10, 1, device=gpu)),
                dict(add=torch.zeros(1, 20, device=gpu).expand(10, 20)),
                dict(out=x.reshape(-1)[:200].reshape(20, 10).t())):
        with pytest.raises(octnca.OctreeNCAError):
            drop(x, **{"out": torch.zeros_like(x), **bad})
    buf = torch.zeros(10, 30, device=gpu)
    with pytest.raises(octnca.OctreeNCAError):
        drop(buf[:, :20], buf[:, 5:25])
    for rate in (-0.1, 1.5, float("nan")):
        with pytest.raises(octnca.OctreeNCAError):
            Dropout(rate, 1)(x, torch.zeros_like(x))
    with pytest.raises(octnca.OctreeNCAError):
        Dropout(0.5, 1, torch.zeros(2, dtype=torch.int64, device=gpu))(x, torch.zeros_like(x))
