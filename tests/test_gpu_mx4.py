"""Matrices in microscaled 4 bits on the GPU: codes and values against the plain
definition, products and gradients against 64 bits.

Tolerances.  Codes and values are exact.  A product's terms are exact (a code has
two significant bits), so only sums and the last rounding err: K terms and the
bias, in any order, each addition off by at most 2^-23 (cut off or rounded) of
the sum of magnitudes S so far, plus half a step of out's type, plus what fp32
cannot hold below 2^-126.  Gradients likewise, with three bf16 parts to a term."""
import numpy as np
import pytest
import torch

import cells4
import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import CellLayer, MX4Matrix

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}   # smallest steps


def spaced(x, pad, fill=7.0):
    """x with its rows `pad` values apart, and the buffer that holds them."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]], wide


def values_of(m):
    out = torch.empty((m.used, m.cols), device="cuda")
    return m.dequantise(out).double()


def sum_bound(terms, magnitudes, result, dtype):
    """Bound of the error of `result`, sums of `terms` exact terms whose magnitudes
    add up to `magnitudes`."""
    return ((terms + 2) * 2.0 ** -23 * magnitudes + terms * 2.0 ** -126 +
            torch.finfo(TYPES[dtype]).eps / 2 * result.abs() * (1 + 2.0 ** -10) + TINY[dtype])


def check(got, want, bound):
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    worst = (err / bound).max().item()
    assert worst <= 1.0, f"error is {worst} of its bound"


def special(rows, cols, seed):
    """Values of every kind: ties, the borders of scales, subnormal and huge ones."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 6, (rows, 1))
    grid = rng.choice([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6],
                      (rows, cols)) * rng.choice([-1, 1], (rows, cols))
    kind = rng.integers(0, 6, rows)
    x[kind == 1] = grid[kind == 1]
    x[kind == 2] = 0.0
    x[kind == 3] = (grid * 2.0 ** -136)[kind == 3]
    x[kind == 4] = (grid * 2.0 ** 125)[kind == 4]
    return x


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 32, 0), (3, 5, 0), (15, 31, 2),
                                           (16, 33, 0), (17, 64, 8), (40, 100, 4), (9, 517, 0),
                                           (70, 40, 1), (5, 1000, 24)])
def test_quantise(gpu, dtype, rows, cols, pad):
    x = torch.from_numpy(special(rows, cols, rows * cols)).to(gpu, TYPES[dtype])
    if dtype == "f16":
        x = x.clamp(-6e4, 6e4)
    shapes = octnca.mx4_shapes(rows, cols)
    m = MX4Matrix(rows, cols, torch.full(shapes[0], 0xA5, dtype=torch.uint8, device=gpu),
                  torch.full(shapes[1], 0x5A, dtype=torch.uint8, device=gpu))
    m.quantise(spaced(x, pad)[0])
    values, codes, scales = cells4.quantise(x.double().cpu().numpy())
    want_c, want_s = cells4.packed(codes, scales)
    row = np.arange(want_s.shape[0] * 16).reshape(-1, 1, 16)
    live = np.broadcast_to(row < rows, want_s.shape)
    got_c, got_s = m.buffers.codes.cpu().numpy(), m.buffers.scales.cpu().numpy()
    # rows past the last are left as they were
    assert np.array_equal(got_s, np.where(live, want_s, 0x5A))
    assert np.array_equal(got_c, np.where(live[..., None], want_c, 0xA5))
    for back in TYPES.values():
        out, wide = spaced(torch.zeros((rows, cols), dtype=back, device=gpu), pad)
        m.dequantise(out)
        assert torch.equal(out, torch.from_numpy(values).to(gpu).to(torch.float32).to(back))
        assert (wide[:, cols:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_blocks_that_are_not_finite(gpu, dtype):
    x = torch.randn(20, 70, device=gpu).to(TYPES[dtype])
    x[3, 40] = float("nan")
    x[7, 0] = float("inf")
    x[16, 69] = -float("inf")
    m = MX4Matrix(20, 70).quantise(x)
    values = values_of(m)
    want = torch.from_numpy(cells4.quantise(x.double().cpu().numpy())[0]).to(gpu)
    assert torch.equal(values.isnan(), want.isnan()) and int(values.isnan().sum()) == 32 + 32 + 6
    assert torch.equal(values.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("rows", [1, 16, 33, 200, 5000])
@pytest.mark.parametrize("relu", [False, True])
def test_product_with_nan_blocks(gpu, rows, relu):
    """They reach every output of their row, or of their weight's column, and no
    other."""
    for outs, cols in ((5, 20), (40, 64), (130, 300)):
        x, w = torch.randn(rows, cols, device=gpu), torch.randn(outs, cols, device=gpu)
        x[rows // 2, cols - 1] = float("nan")
        w[outs // 3, 0] = float("inf")
        layer = CellLayer(w, rows=rows)
        out = layer.forward(x, torch.zeros(rows, outs, device=gpu), relu=relu)
        bad = torch.zeros(rows, outs, dtype=torch.bool, device=gpu)
        bad[rows // 2] = True
        bad[:, outs // 3] = True
        assert torch.equal(out.isnan(), bad)
        again = layer.forward(layer.kept, torch.zeros(rows, outs, device=gpu), relu=relu)
        assert torch.equal(again.isnan(), bad)


SIZES = [  # rows, cols, outs: one cell, few, many; parts of blocks and groups
    (1, 1, 1), (1, 32, 16), (1, 4096, 64), (1, 1000, 1003), (2, 517, 33), (5, 64, 300),
    (16, 2048, 100), (17, 96, 16), (33, 128, 129), (64, 33, 2), (100, 300, 70), (257, 128, 256),
    (300, 1024, 520), (1000, 16, 19), (1031, 20, 100), (5000, 32, 64), (3001, 40, 3),
    (20011, 64, 16), (4099, 100, 20), (513, 640, 600), (70001, 32, 2),
    # each way to share few rows out; as many values as a workgroup quantises, and more
    (40, 1000, 300), (20, 1000, 300), (20, 1100, 4099), (50, 1100, 4099), (5, 5, 300),
    (3, 7, 1000), (16, 1024, 300), (17, 1024, 300), (15, 1056, 300), (200, 3, 140)]


@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_product(gpu, rows, cols, outs):
    rng = np.random.default_rng(rows + cols + outs)
    gen = torch.Generator(device=gpu).manual_seed(rows * 7 + cols * 3 + outs)
    x = torch.randn(rows, cols, generator=gen, device=gpu)
    x *= torch.exp2(torch.randint(-8, 8, (rows, 1), generator=gen, device=gpu).float())
    w = torch.randn(outs, cols, generator=gen, device=gpu)
    for dtype, out_type, pad, with_bias, relu in (
            ("f32", "f32", 0, True, False), ("bf16", "bf16", 0, False, True),
            ("f16", "f32", int(rng.integers(1, 9)), True, True), ("f32", "f16", 4, False, False),
            ("bf16", "f32", 8, True, False)):
        bias = torch.randn(outs, generator=gen, device=gpu) if with_bias else None
        layer = CellLayer(w, bias, rows=rows)
        out, wide = spaced(torch.zeros((rows, outs), dtype=TYPES[out_type], device=gpu), pad)
        layer.forward(spaced(x.to(TYPES[dtype]), pad)[0], out, relu=relu)
        # the codes are those of a quantisation alone
        alone = MX4Matrix(rows, cols).quantise(x.to(TYPES[dtype]))
        a, v = values_of(layer.kept), values_of(layer.w)
        assert torch.equal(a, values_of(alone))
        want, mags = a @ v.t(), a.abs() @ v.abs().t()
        if bias is not None:
            want, mags = want + bias, mags + bias.abs()
        if relu:
            want = want.clamp(min=0)
        if out_type == "f16":
            assert want.abs().max() < 6e4
        bound = sum_bound(cols, mags, want, out_type)
        check(out, want, bound)
        again, wide2 = spaced(torch.zeros_like(out, memory_format=torch.contiguous_format), pad)
        layer.forward(layer.kept, again, relu=relu)
        check(again, want, bound)
        assert (wide[:, outs:] == 7).all() and (wide2[:, outs:] == 7).all()
        # the same call, the same bits
        repeat = torch.zeros_like(out)
        layer.forward(spaced(x.to(TYPES[dtype]), pad)[0], repeat, relu=relu)
        assert torch.equal(repeat, out)


@pytest.mark.parametrize("rows,cols,outs", [(4096, 4096, 512), (300, 20000, 300), (1, 70000, 5),
                                            (900_001, 32, 64), (1100, 2080, 1050)])
def test_large_product(gpu, rows, cols, outs):
    gen = torch.Generator(device=gpu).manual_seed(5)
    x = torch.randn(rows, cols, generator=gen, device=gpu, dtype=torch.bfloat16)
    layer = CellLayer(torch.randn(outs, cols, generator=gen, device=gpu), rows=rows)
    out = layer.forward(x, torch.zeros(rows, outs, device=gpu))
    a, v = values_of(layer.kept), values_of(layer.w)
    want = a @ v.t()
    check(out, want, sum_bound(cols, a.abs() @ v.abs().t(), want, "f32"))


def test_no_rows(gpu):
    layer = CellLayer(torch.randn(4, 40, device=gpu), torch.randn(4, device=gpu), rows=8, train=True)
    out = torch.zeros(0, 4, device=gpu)
    layer.forward(torch.zeros(0, 40, device=gpu), out)
    layer.grad_weight.fill_(3.0)
    layer.grad_bias.fill_(3.0)
    layer.backward(out, torch.zeros(0, 40, device=gpu))
    assert (layer.grad_weight == 0).all() and (layer.grad_bias == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", [(1, 1, 1), (1, 100, 30), (2, 517, 33), (17, 96, 16),
                                            (63, 33, 65), (100, 300, 70), (1000, 16, 19),
                                            (1031, 20, 100), (5003, 32, 64), (20011, 64, 16),
                                            (700, 640, 600), (130, 1100, 257), (40000, 40, 3),
                                            (3, 9, 7), (50, 130, 5), (633, 10, 925),
                                            (2000, 128, 60), (2000, 60, 128), (999, 128, 128)])
def test_backward(gpu, rows, cols, outs, dtype):
    gen = torch.Generator(device=gpu).manual_seed(rows * 5 + cols + outs)
    g = torch.randn(rows, outs, generator=gen, device=gpu)
    g *= torch.exp2(torch.randint(-9, 3, (rows, 1), generator=gen, device=gpu).float())
    g = g.to(TYPES[dtype])
    layer = CellLayer(torch.randn(outs, cols, generator=gen, device=gpu),
                      torch.zeros(outs, device=gpu), rows=rows, train=True)
    layer.kept.quantise(torch.randn(rows, cols, generator=gen, device=gpu))
    a, v, gd = values_of(layer.kept), values_of(layer.w), g.double()
    for pad in (0, 3, 8):
        grad_in, wide = spaced(torch.zeros((rows, cols), dtype=TYPES[dtype], device=gpu), pad)
        layer.grad_weight.fill_(9.0)
        layer.grad_bias.fill_(9.0)
        layer.backward(spaced(g, pad)[0], grad_in)
        want = gd @ v
        check(grad_in, want, sum_bound(3 * outs, gd.abs() @ v.abs(), want, dtype))
        want = gd.t() @ a
        check(layer.grad_weight, want, sum_bound(3 * rows, gd.abs().t() @ a.abs(), want, "f32"))
        want = gd.sum(0)
        check(layer.grad_bias, want, sum_bound(rows, gd.abs().sum(0), want, "f32"))
        assert (wide[:, cols:] == 7).all()
        first = layer.grad_weight.clone(), layer.grad_bias.clone(), grad_in.clone()
        layer.backward(spaced(g, pad)[0], grad_in)
        assert all(torch.equal(x, y) for x, y in
                   zip(first, (layer.grad_weight, layer.grad_bias, grad_in)))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,outs,pad", [(300, 3500, 3700, 0), (13001, 1030, 133, 0),
                                                (500, 3584, 3600, 1)])
def test_large_backward(gpu, rows, cols, outs, dtype, pad):
    gen = torch.Generator(device=gpu).manual_seed(rows)
    g = torch.randn(rows, outs, generator=gen, device=gpu).to(TYPES[dtype])
    layer = CellLayer(torch.randn(outs, cols, generator=gen, device=gpu),
                      torch.zeros(outs, device=gpu), rows=rows, train=True)
    layer.kept.quantise(torch.randn(rows, cols, generator=gen, device=gpu))
    a, v, gd = values_of(layer.kept), values_of(layer.w), g.double()
    grad_in, wide = spaced(torch.zeros((rows, cols), dtype=TYPES[dtype], device=gpu), pad)
    layer.backward(spaced(g, pad)[0], grad_in)
    want = gd @ v
    check(grad_in, want, sum_bound(3 * outs, gd.abs() @ v.abs(), want, dtype))
    want = gd.t() @ a
    check(layer.grad_weight, want, sum_bound(3 * rows, gd.abs().t() @ a.abs(), want, "f32"))
    want = gd.sum(0)
    check(layer.grad_bias, want, sum_bound(rows, gd.abs().sum(0), want, "f32"))
    assert (wide[:, cols:] == 7).all()


@pytest.mark.parametrize("rows,cols,outs", [(900, 70, 50), (900, 200, 150), (300, 3500, 3700)])
def test_backward_parts(gpu, rows, cols, outs):
    """Each gradient alone gives the bits that all together give."""
    layer = CellLayer(torch.randn(outs, cols, device=gpu), rows=rows, train=True)
    layer.kept.quantise(torch.randn(rows, cols, device=gpu))
    g = torch.randn(rows, outs, device=gpu)
    new = lambda: (torch.full((rows, cols), 5.0, device=gpu),
                   torch.full((outs, cols), 5.0, device=gpu), torch.full((outs,), 5.0, device=gpu))
    whole = new()
    call = lambda i, w, b: octnca.octree_nca_mx4_backward(g, layer.kept.struct, layer.w.struct, i,
                                                          w, b, layer.workspace)
    call(*whole)
    for mask in range(8):
        part = new()
        call(*(t if mask >> k & 1 else None for k, t in enumerate(part)))
        for k in range(3):
            assert torch.equal(part[k], whole[k]) if mask >> k & 1 else (part[k] == 5).all()
    octnca.octree_nca_mx4_backward(g, layer.kept.struct, layer.w.struct, whole[0])


def test_backward_values_that_are_not_finite(gpu):
    """An infinite gradient gives infinities of the right sign, a NaN NaNs, in its
    own row and column; fp32's largest values stay finite where they can."""
    layer = CellLayer(torch.randn(40, 64, device=gpu).sign(), rows=100, train=True)
    layer.kept.quantise(torch.randn(100, 64, device=gpu).sign())
    g = torch.randn(100, 40, device=gpu)
    g[10, 3], g[20, 5], g[30, 7] = float("inf"), float("nan"), 3.4e38
    a, v = values_of(layer.kept), values_of(layer.w)
    grad_in = torch.zeros(100, 64, device=gpu)
    layer.backward(g, grad_in)
    want_in, want_w = g.double() @ v, g.double().t() @ a
    for got, want in ((grad_in, want_in), (layer.grad_weight, want_w)):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
        assert torch.equal(got[want.isinf()] > 0, want[want.isinf()] > 0)
        ok = want.isfinite()
        assert ((got.double() - want)[ok].abs() <= 1e-4 * (1 + want[ok].abs())).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", [(300, 70, 40), (300, 300, 200), (300, 3500, 3700)])
def test_backward_with_odd_blocks(gpu, rows, cols, outs, dtype):
    """Blocks of NaN reach the gradients of their columns and no others; blocks of the
    smallest and of large scales are exact."""
    w, x = torch.randn(outs, cols, device=gpu), torch.randn(rows, cols, device=gpu)
    w[3, :32] *= 2.0 ** -126       # scale 2^-127: what is left of it is below 2^-124
    x[5, 32:64] *= 2.0 ** 100
    w[outs - 1, cols - 1] = float("nan")
    x[rows - 1, 33] = float("inf")
    layer = CellLayer(w, rows=rows, train=True)
    layer.kept.quantise(x)
    g = torch.randn(rows, outs, device=gpu).to(TYPES[dtype])
    grad_in = torch.zeros((rows, cols), dtype=TYPES[dtype], device=gpu)
    layer.backward(g, grad_in)
    a, v, gd = values_of(layer.kept), values_of(layer.w), g.double()
    nan_in = torch.zeros(cols, dtype=torch.bool, device=gpu)
    nan_in[(cols - 1) // 32 * 32:] = True
    nan_w = torch.zeros(cols, dtype=torch.bool, device=gpu)
    nan_w[32:64] = True
    assert torch.equal(grad_in.isnan(), nan_in.expand(rows, cols))
    assert torch.equal(layer.grad_weight.isnan(), nan_w.expand(outs, cols))
    want = (gd @ v.nan_to_num())[:, ~nan_in]
    check(grad_in[:, ~nan_in], want,
          sum_bound(3 * outs, (gd.abs() @ v.nan_to_num().abs())[:, ~nan_in], want, dtype))
    want = (gd.t() @ a.nan_to_num())[:, ~nan_w]
    check(layer.grad_weight[:, ~nan_w], want,
          sum_bound(3 * rows, (gd.abs().t() @ a.nan_to_num().abs())[:, ~nan_w], want, "f32"))


def test_gradients_by_differences(gpu):
    """grad_weight and grad_in against difference quotients of the product itself:
    it is linear in each code's value, and steps of whole values keep the scales."""
    rng = np.random.default_rng(0)
    grid = np.array([-6, -4, -3, -2, -1.5, -1, -0.5, 0.5, 1, 1.5, 2, 3, 4, 6])
    w, x = (torch.tensor(rng.choice(grid, s), device=gpu, dtype=torch.float32)
            for s in ((9, 40), (30, 40)))
    w[:, ::32], x[:, ::32] = 6.0, 6.0     # every block's largest
    g = torch.tensor(rng.integers(-8, 9, (30, 9)), device=gpu, dtype=torch.float32)
    layer = CellLayer(w, rows=30, train=True)
    out = torch.zeros(30, 9, device=gpu)
    grad_in = torch.zeros(30, 40, device=gpu)

    def loss():
        layer.refresh()
        layer.forward(x, out)
        return (out.double() * g.double()).sum().item()
    loss()
    layer.backward(g, grad_in)
    for t, grad in ((w, layer.grad_weight), (x, grad_in)):
        for _ in range(25):
            i, j = rng.integers(t.shape[0]), rng.integers(1, 32)
            old = t[i, j].item()
            t[i, j] = 2.0
            up = loss()
            t[i, j] = -2.0
            down = loss()
            t[i, j] = old
            assert (up - down) / 4.0 == grad[i, j].item()


def test_columns_of_one_buffer(gpu):
    """Inputs, outputs and gradients that are columns of one buffer."""
    buf = torch.randn(50, 100, device=gpu)
    layer = CellLayer(torch.randn(20, 40, device=gpu), rows=50, train=True)
    want = layer.forward(buf[:, 5:45].contiguous(), torch.zeros(50, 20, device=gpu))
    before = buf.clone()
    layer.forward(buf[:, 5:45], buf[:, 45:65])
    assert torch.equal(buf[:, 45:65], want)
    grad_in = torch.zeros(50, 40, device=gpu)
    layer.backward(buf[:, 45:65].contiguous(), grad_in)
    layer.backward(buf[:, 45:65], buf[:, 5:45])
    assert torch.equal(buf[:, 5:45], grad_in)
    assert torch.equal(buf[:, 65:], before[:, 65:]) and torch.equal(buf[:, :5], before[:, :5])
    with pytest.raises(octnca.OctreeNCAError):
        layer.forward(buf[:, 5:45], buf[:, 40:60])


def test_fewer_rows_than_room(gpu):
    layer = CellLayer(torch.randn(20, 40, device=gpu), torch.randn(20, device=gpu), rows=500,
                      train=True)
    for n in (500, 1, 37):
        x, g = torch.randn(n, 40, device=gpu), torch.randn(n, 20, device=gpu)
        out, grad_in = torch.zeros(n, 20, device=gpu), torch.zeros(n, 40, device=gpu)
        layer.forward(x, out)
        layer.backward(g, grad_in)
        a, v = values_of(layer.kept), values_of(layer.w)
        assert a.shape == (n, 40)
        want = a @ v.t() + layer.bias
        check(out, want, sum_bound(40, a.abs() @ v.abs().t() + layer.bias.abs(), want, "f32"))
        want = g.double().t() @ a
        check(layer.grad_weight, want,
              sum_bound(3 * n, g.double().abs().t() @ a.abs(), want, "f32"))
    with pytest.raises(octnca.OctreeNCAError):
        layer.forward(torch.zeros(501, 40, device=gpu), torch.zeros(501, 20, device=gpu))
    with pytest.raises(octnca.OctreeNCAError):   # not the rows of the last forward
        layer.backward(torch.zeros(36, 20, device=gpu))
    # a refused call leaves the last forward's rows
    with pytest.raises(octnca.OctreeNCAError):
        layer.forward(torch.zeros(5, 40, device=gpu), torch.zeros(4, 20, device=gpu))
    with pytest.raises(octnca.OctreeNCAError):
        layer.kept.quantise(torch.zeros(5, 41, device=gpu))
    assert layer.kept.used == 37


@pytest.mark.parametrize("rows,cols,outs", [(5, 40, 20), (5, 300, 200), (37, 300, 200),
                                            (1100, 40, 20), (5003, 200, 1500)])
def test_memory_past_the_rows_is_left(gpu, rows, cols, outs):
    """The input's codes, however the product is made, and the outputs' buffer."""
    layer = CellLayer(torch.randn(outs, cols, device=gpu), rows=rows)
    codes, scales = layer.kept.buffers.codes, layer.kept.buffers.scales
    codes.fill_(0xA5)
    scales.fill_(0x5A)
    out = torch.full((rows + 3, outs), 7.0, device=gpu)
    layer.forward(torch.randn(rows, cols, device=gpu), out[:rows])
    past = torch.arange(codes.shape[0] * 16, device=gpu).reshape(-1, 1, 16) >= rows
    past = past.expand(scales.shape)
    assert (scales[past] == 0x5A).all() and (codes[past] == 0xA5).all()
    assert (scales[~past] != 0x5A).all() and (out[rows:] == 7).all()
    assert torch.equal(values_of(layer.kept).isfinite().all(), torch.tensor(True, device=gpu))


def test_states_and_images_as_rows(gpu):
    """Tensors of more dimensions are taken by their last."""
    state = torch.randn(1, 12, 20, 16, device=gpu)
    layer = CellLayer(torch.randn(5, 16, device=gpu), rows=240)
    a = layer.forward(state, torch.zeros(1, 12, 20, 5, device=gpu))
    b = layer.forward(state.reshape(240, 16), torch.zeros(240, 5, device=gpu))
    assert torch.equal(a.reshape(240, 5), b)


def test_far_rows(gpu):
    """Codes and values past 2^32 bytes: the last rows as in a matrix of their own."""
    rows, cols, few = 4_300_003, 2100, 83          # codes 4.5 GB, values 18 GB
    first = rows // 16 * 16 - 64                   # whole row groups before the last ones
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=gpu)
    x[:1000].normal_()
    x[1000:first] = 0
    x[first:].normal_()
    layer = CellLayer(torch.randn(20, cols, device=gpu), rows=rows, train=True)
    assert layer.kept.buffers.codes.numel() > 2 ** 32
    alone = CellLayer(layer.weight, rows=few, train=True)
    out = layer.forward(x, torch.empty((rows, 20), device=gpu))
    last, n = x[first:], rows - first
    want = alone.forward(last, torch.empty((n, 20), device=gpu))
    a, v = values_of(alone.kept), values_of(alone.w)
    groups = layer.kept.buffers.codes[first // 16:], layer.kept.buffers.scales[first // 16:]
    assert torch.equal(groups[0][:4], alone.kept.buffers.codes[:4])
    assert torch.equal(groups[1][:4], alone.kept.buffers.scales[:4])
    exact = a @ v.t()
    bound = sum_bound(cols, a.abs() @ v.abs().t(), exact, "f32")
    check(out[first:], exact, bound)
    check(want, exact, bound)
    assert (out[1000:first] == 0).all()
    back = layer.kept.dequantise(torch.empty_like(x))
    assert torch.equal(back[first:].double(), a) and (back[1000:first] == 0).all()
    del back
    g = torch.zeros((rows, 20), device=gpu)
    g[first:].normal_()
    grad_in = torch.empty_like(x, dtype=torch.float32)
    layer.backward(g, grad_in)
    gd = g[first:].double()
    exact = gd @ v
    check(grad_in[first:], exact, sum_bound(60, gd.abs() @ v.abs(), exact, "f32"))
    assert (grad_in[:first] == 0).all()
    exact = gd.t() @ a     # the other rows' terms are zeros
    check(layer.grad_weight, exact, sum_bound(3 * n + 512, gd.abs().t() @ a.abs(), exact, "f32"))
