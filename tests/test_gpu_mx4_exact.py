"""Products and gradients of cell layers where nothing may be lost: sums that are exact
in fp32 in any order, and gradients of one term, all bits of which come back.

Values are those of the 4-bit grid with scale 1, so a product's terms are multiples of
1/4 up to 36, and a gradient's, with whole numbers up to 8 in G, multiples of 1/2 up to
48: any sum of fewer than 2^24 / 144, or 2^24 / 96, of them is a multiple of its unit
below 2^24 units, which fp32 holds.  So the result is the same whatever the order, and a
term left out or taken twice shows."""
import pytest
import torch

from paper_2508_06993_amd.runtime import CellLayer

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GRID = (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
POWERS = (0.5, 1.0, 2.0, 4.0)


def on_grid(rows, cols, gen, levels=GRID):
    """Values of the grid, none of them 0; every block of 32 has the largest level."""
    device = gen.device
    table = torch.tensor(levels, device=device)
    x = table[torch.randint(len(levels), (rows, cols), generator=gen, device=device)]
    x[:, ::32] = levels[-1]
    return x * (torch.randint(2, (rows, cols), generator=gen, device=device) * 2 - 1)


def held(m):
    return m.dequantise(torch.empty((m.used, m.cols), device="cuda"))


PRODUCTS = [  # rows, cols, outs
    (1, 1, 1), (1, 4096, 64), (1, 1000, 1003), (1, 70000, 5), (2, 517, 33), (5, 64, 300),
    (8, 16400, 1000), (16, 2048, 100), (16, 4100, 2100), (17, 96, 16), (17, 1100, 4099),
    (33, 128, 129), (40, 1000, 300), (50, 1100, 4099), (64, 33, 2), (100, 300, 70),
    (300, 1024, 520), (300, 20000, 300), (1000, 16, 19), (1000, 517, 1003), (1031, 20, 100),
    (5000, 32, 64), (20011, 64, 16), (4099, 100, 20), (3001, 128, 128), (1100, 2080, 1050),
    (4096, 4096, 512), (4100, 610, 4100), (900_001, 32, 64),
    # each number of waves, for each number of rows that they take
    (16, 1024, 4096), (4, 1030, 1000), (16, 1024, 4100), (1, 8200, 2000), (20, 6200, 1000),
    (20, 4100, 1000), (30, 1000, 1003), (40, 16400, 300), (64, 16300, 300), (1, 300, 4099),
    # both sides of the number of tiles from which they are taken
    (512, 1530, 4096), (512, 1540, 4096), (640, 1540, 4096), (1020, 300, 1920), (65, 300, 16384),
    (1030, 1540, 1920), (10300, 1540, 3), (16300, 1540, 100)]


@pytest.mark.parametrize("rows,cols,outs", PRODUCTS)
def test_products(gpu, rows, cols, outs):
    assert cols * 144 < 2 ** 24
    gen = torch.Generator(device=gpu).manual_seed(rows + 3 * cols + 7 * outs)
    x, w = on_grid(rows, cols, gen), on_grid(outs, cols, gen)
    bias = torch.randint(-100, 100, (outs,), generator=gen, device=gpu).float()
    layer = CellLayer(w, bias, rows=rows)
    assert torch.equal(held(layer.w), w)
    want = x.double() @ w.double().t() + bias
    for dtype, out_type, relu in (("f32", "f32", False), ("bf16", "f32", False),
                                  ("f16", "bf16", True), ("f32", "f16", False)):
        # exact in fp32, so rounded once on the way to 16 bits
        expect = (want.clamp(min=0) if relu else want).float().to(TYPES[out_type])
        new = lambda: torch.full((rows, outs), 7.0, dtype=TYPES[out_type], device=gpu)
        out = layer.forward(x.to(TYPES[dtype]), new(), relu=relu)
        assert torch.equal(held(layer.kept), x)
        assert torch.equal(out, expect)
        assert torch.equal(layer.forward(layer.kept, new(), relu=relu), expect)


GRADIENTS = [  # rows, cols, outs
    (1, 1, 1), (1, 100, 30), (2, 517, 33), (17, 96, 16), (63, 33, 65), (1000, 16, 19),
    (1031, 20, 100), (5003, 32, 64), (102_401, 32, 64), (20011, 64, 16), (2000, 128, 60),
    (2000, 60, 128), (999, 128, 128), (40000, 40, 3), (100_003, 100, 30), (700, 640, 600),
    (130, 1100, 257), (1000, 517, 1003), (13001, 1030, 133), (100_000, 300, 40),
    (300, 3500, 3700), (500, 3584, 3600), (6000, 4096, 4100),
    # both sides of the number of tiles up to which grad_in takes small ones
    (1000, 1024, 1024), (2030, 1000, 500), (2060, 1000, 131)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", GRADIENTS)
def test_gradients(gpu, rows, cols, outs, dtype):
    assert max(rows, outs) * 96 < 2 ** 24
    gen = torch.Generator(device=gpu).manual_seed(rows + 3 * cols + 7 * outs)
    x, w = on_grid(rows, cols, gen), on_grid(outs, cols, gen)
    layer = CellLayer(w, torch.zeros(outs, device=gpu), rows=rows, train=True)
    layer.kept.quantise(x)
    g = torch.randint(1, 9, (rows, outs), generator=gen, device=gpu).to(TYPES[dtype])
    g *= torch.randint(2, (rows, outs), generator=gen, device=gpu) * 2 - 1
    grad_in = torch.full((rows, cols), 7.0, dtype=TYPES[dtype], device=gpu)
    layer.grad_weight.fill_(7.0)
    layer.grad_bias.fill_(7.0)
    layer.backward(g, grad_in)
    gd = g.double()
    assert torch.equal(grad_in, (gd @ w.double()).float().to(TYPES[dtype]))
    assert torch.equal(layer.grad_weight, (gd.t() @ x.double()).float())
    assert torch.equal(layer.grad_bias, gd.sum(0).float())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", GRADIENTS)
def test_gradients_of_one_term(gpu, rows, cols, outs, dtype):
    """G has one value at most in a row and a column, of all the bits of its type, and
    the codes are powers of two: each product is a value of G's type."""
    gen = torch.Generator(device=gpu).manual_seed(rows + 5 * cols + 11 * outs)
    x, w = on_grid(rows, cols, gen, POWERS), on_grid(outs, cols, gen, POWERS)
    layer = CellLayer(w, torch.zeros(outs, device=gpu), rows=rows, train=True)
    layer.kept.quantise(x)
    n = min(rows, outs)
    at = torch.randperm(rows, generator=gen, device=gpu)[:n]
    to = torch.randperm(outs, generator=gen, device=gpu)[:n]
    bits = {"f32": 23, "f16": 10, "bf16": 7}[dtype]
    value = 1 + torch.randint(2 ** bits, (n,), generator=gen, device=gpu) * 2.0 ** -bits
    value *= torch.exp2(torch.randint(-2, 4, (n,), generator=gen, device=gpu).float())
    value *= torch.randint(2, (n,), generator=gen, device=gpu) * 2 - 1
    g = torch.zeros((rows, outs), dtype=TYPES[dtype], device=gpu)
    g[at, to] = value.to(TYPES[dtype])
    assert torch.equal(g[at, to].float(), value)
    grad_in = torch.full((rows, cols), 7.0, dtype=TYPES[dtype], device=gpu)
    layer.backward(g, grad_in)
    want_in, want_weight = torch.zeros(rows, cols, device=gpu), torch.zeros(outs, cols, device=gpu)
    want_in[at] = value[:, None] * w[to]
    want_weight[to] = value[:, None] * x[at]
    want_bias = torch.zeros(outs, device=gpu)
    want_bias[to] = value
    assert torch.equal(grad_in.float(), want_in)
    assert torch.equal(layer.grad_weight, want_weight)
    assert torch.equal(layer.grad_bias, want_bias)
