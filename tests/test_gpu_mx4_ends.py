"""Matrices in 4 bits at both ends of fp32's range.  Products take the codes and scales
as they are, so their terms are exact where fp32 holds them; gradients take values in
bf16, where 2^128 is infinite."""
import pytest
import torch

from paper_2508_06993_amd.runtime import CellLayer, MX4Matrix

pytestmark = pytest.mark.gpu

# each way a product is made
SIZES = [(5, 64, 20), (1, 300, 300), (5, 3000, 300), (300, 300, 200), (1100, 2080, 1050),
         (4100, 300, 4100)]


@pytest.mark.parametrize("largest", [3.4e38, 1.75 * 2.0 ** 127, 1.7499 * 2.0 ** 127])
def test_largest_values_read_back(gpu, largest):
    """Steps above 1.5 * 2^127 are 2^126: from 1.75 * 2^127 on the nearest value (the
    even code of two) is 2^128."""
    x = torch.full((1, 40), 1.0, device=gpu)
    x[0, 3], x[0, 4] = largest, -largest
    m = MX4Matrix(1, 40).quantise(x)
    up = largest >= 1.75 * 2.0 ** 127
    assert m.buffers.scales[0, 0, 0] == 253
    assert m.buffers.codes[0, 0, 0, 1:3].tolist() == ([6 << 4, 14] if up else [5 << 4, 13])
    want = torch.zeros(1, 40)
    want[0, 32:] = 1.0
    want[0, 3] = float("inf") if up else 1.5 * 2.0 ** 127
    want[0, 4] = -want[0, 3]
    for dtype in (torch.float32, torch.bfloat16):
        out = m.dequantise(torch.zeros(1, 40, dtype=dtype, device=gpu))
        assert torch.equal(out.cpu(), want.to(dtype))


@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_products_take_2_128(gpu, rows, cols, outs):
    x, w = torch.zeros(rows, cols, device=gpu), torch.ones(outs, cols, device=gpu) * 2.0 ** -60
    x[:, cols - 1] = 3.4e38
    layer = CellLayer(w, rows=rows)
    new = lambda: torch.zeros(rows, outs, device=gpu)
    assert (layer.forward(x, new()) == 2.0 ** 68).all()
    assert (layer.forward(layer.kept, new()) == 2.0 ** 68).all()


@pytest.mark.parametrize("rows,cols,outs", SIZES)
@pytest.mark.parametrize("ex,ew", [(-70, -60), (-127, 0), (-127, -10), (-100, -47)])
def test_small_products(gpu, rows, cols, outs, ex, ew):
    """One term, a multiple of 2^-147 or more: exact, below fp32's normal numbers too."""
    x, w = torch.zeros(rows, cols, device=gpu), torch.zeros(outs, cols, device=gpu)
    codes = torch.arange(rows, device=gpu) % 4 + 1.0
    x[:, cols - 1] = (codes.double() * 2.0 ** ex).float()
    w[:, cols - 1] = 2.0 ** ew
    layer = CellLayer(w, rows=rows)
    out = layer.forward(x, torch.zeros(rows, outs, device=gpu))
    want = (codes.double() * 2.0 ** (ex + ew)).float()
    assert torch.equal(out, want[:, None].expand(rows, outs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,outs", [(300, 64, 40), (300, 300, 200), (300, 3500, 3700)])
def test_gradients_of_2_128_are_not_finite(gpu, rows, cols, outs, dtype):
    """In its own columns, and only there."""
    x, w = torch.ones(rows, cols, device=gpu), torch.ones(outs, cols, device=gpu)
    x[7, 5], w[9, 33] = 3.4e38, -3.4e38
    layer = CellLayer(w, rows=rows, train=True)
    layer.kept.quantise(x)
    g = torch.ones(rows, outs, device=gpu).to(dtype)
    g[7, 0], g[0, 9] = 0.0, 0.0
    grad_in = torch.zeros(rows, cols, device=gpu, dtype=dtype)
    layer.backward(g, grad_in)
    column = torch.arange(cols, device=gpu)
    assert torch.equal(layer.grad_weight.isfinite(), (column != 5).expand(outs, cols))
    assert torch.equal(grad_in.isfinite(), (column != 33).expand(rows, cols))
