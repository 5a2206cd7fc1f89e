"""Memory of cell layers across streams: what a call reads on another stream is not
handed out again before the call is done."""
import contextlib

import pytest
import torch

from paper_2508_06993_amd.runtime import CellLayer, MX4Matrix

pytestmark = pytest.mark.gpu

ROWS, COLS, OUTS = 4000, 200, 70


def busy(stream):
    """Some tens of milliseconds of work."""
    with torch.cuda.stream(stream):
        a = torch.randn(4096, 4096, device="cuda") / 64
        for _ in range(30):
            a = a @ a / 64


def overwrite(matrix_bytes):
    """Takes what memory the allocator has of these sizes and fills it."""
    return [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
            for n in matrix_bytes for _ in range(4)]


@pytest.mark.parametrize("kind", ["object", "current"])
@pytest.mark.parametrize("way", ["forward", "backward"])
def test_a_given_matrix_may_be_dropped(gpu, kind, way):
    x = torch.randn(ROWS, COLS, device=gpu)
    g = torch.randn(ROWS, OUTS, device=gpu)
    layer = CellLayer(torch.randn(OUTS, COLS, device=gpu), rows=ROWS, train=True)
    want = layer.forward(MX4Matrix(ROWS, COLS).quantise(x), torch.zeros(ROWS, OUTS, device=gpu))
    layer.backward(g)
    want_weight = layer.grad_weight.clone()
    out = torch.zeros(ROWS, OUTS, device=gpu)
    layer.forward(x, out)           # the layer no longer holds the first matrix
    out.zero_()
    layer.grad_weight.zero_()
    m = MX4Matrix(ROWS, COLS).quantise(x)
    sizes = [m.buffers.codes.numel(), m.buffers.scales.numel()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    context = torch.cuda.stream(side) if kind == "current" else contextlib.nullcontext()
    with context:
        stream = side if kind == "object" else None
        if way == "forward":
            layer.forward(m, out, stream=stream)
        else:
            layer.backward(g, kept=m, stream=stream)
    layer.last = layer.kept         # as a further forward does
    del m
    taken = overwrite(sizes)
    torch.cuda.synchronize()
    assert len(taken) == 8
    if way == "forward":
        assert torch.equal(out, want)
    else:
        assert torch.equal(layer.grad_weight, want_weight)
