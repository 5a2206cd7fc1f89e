"""Cell layers without a GPU: the plain definitions against published answers and
against themselves, and the refusals of the entry points (every call below fails
validation or has nothing to do, so no HIP call is made)."""
import ctypes

import numpy as np
import pytest
import torch

import cells4
import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import _Dropout, _MX4, _Rows

OK, EINVAL, ESHAPE, ESPACE = 0, -1, -3, -5
A, B, D, E, F, G = (0x7f0000000000 + k * 0x100000000 for k in range(6))   # never dereferenced
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib(library_path):
    return octnca.lib()


def test_generator_known_answers():
    """Salmon et al.'s published test vectors of Philox4x32-10."""
    assert cells4.philox4x32([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    m = 0xffffffff
    assert cells4.philox4x32([m] * 4, [m] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_plain_quantise():
    x = np.array([[0.26, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -5.1]])
    values, codes, scales = cells4.quantise(x)
    assert scales[0, 0] == 127
    assert values[0].tolist() == [0.5, 0, 1, 1, 2, 2, 4, 4, 6, -6]
    assert codes[0, 0, :10].tolist() == [1, 0, 2, 2, 4, 4, 6, 6, 7, 15]
    # a scale is the smallest that holds the largest value
    assert cells4.quantise([[6.0001]])[2][0, 0] == 128
    assert cells4.quantise([[3.0]])[2][0, 0] == 126 and cells4.quantise([[0.0]])[2][0, 0] == 0
    assert cells4.quantise([[float(np.finfo(np.float32).max)]])[2][0, 0] == 253
    assert cells4.quantise([[np.inf, 1.0]])[2][0, 0] == 255
    # taken again, values stay
    rng = np.random.default_rng(0)
    v = cells4.quantise(rng.standard_normal((5, 70)))[0]
    assert np.array_equal(cells4.quantise(v)[0], v)


def mx4(rows=20, cols=70, codes=A, scales=B):
    return _MX4(rows, cols, codes, scales)


def rows(data=D, stride=None, dtype=F32, cols=70):
    return _Rows(data, cols if stride is None else stride, dtype)


def test_sizes(lib):
    size = lib.octree_nca_mx4_code_bytes
    assert size(0, 5) == 0 and size(1, 1) == 256 and size(16, 32) == 256
    assert size(17, 33) == 1024 and size(1 << 29, 1 << 20) == 256 << 40
    for bad in ((-1, 4), (4, 0), (4, -1), (4, (1 << 20) + 1), ((1 << 29) + 1, 4)):
        assert size(*bad) == 0, bad
    work = lib.octree_nca_mx4_backward_workspace_bytes
    assert work(0, 4, 4) >= 16
    for bad in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (4, 4, (1 << 20) + 1), ((1 << 29) + 1, 4, 4)):
        assert work(*bad) == 0, bad
    # a smaller call fits the workspace of a larger one
    for cols, outs in ((1, 1), (32, 64), (517, 1003), (4096, 4096)):
        sizes = [work(n, cols, outs) for n in (0, 1, 300, 5000, 100000, 3000000)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("way", ["quantise", "dequantise"])
def test_quantise_refusals(lib, way):
    def call(m, x):
        if way == "quantise":
            return lib.octree_nca_mx4_quantise(x, m, None)
        return lib.octree_nca_mx4_dequantise(m, x, None)
    for m, x in ((None, rows()), (mx4(), None), (mx4(codes=None), rows()),
                 (mx4(scales=None), rows()), (mx4(codes=A + 8), rows()),
                 (mx4(scales=B + 4), rows()), (mx4(scales=A + 64), rows()),
                 (mx4(), rows(None)), (mx4(), rows(D + 2)), (mx4(), rows(D + 1, dtype=BF16)),
                 (mx4(), rows(dtype=3)), (mx4(), rows(dtype=-1)), (mx4(), rows(A + 256)),
                 (mx4(), rows(B - 4))):
        assert call(m, x) == EINVAL
    for m, x in ((mx4(rows=-1), rows()), (mx4(cols=0), rows()), (mx4(cols=1 << 21), rows()),
                 (mx4(rows=1 << 30), rows()), (mx4(), rows(stride=69)), (mx4(), rows(stride=0)),
                 (mx4(), rows(stride=-70)), (mx4(), rows(stride=1 << 60))):
        assert call(m, x) == ESHAPE
    assert call(mx4(rows=0, codes=None, scales=None), rows(None)) == OK


def test_product_refusals(lib):
    def call(a=None, w=None, bias=None, out=None, linear=None):
        a, w = a or mx4(), w or mx4(9, 70, D, E)
        out = out or rows(F, cols=9)
        if linear is not None:
            return lib.octree_nca_mx4_linear(linear, a, w, bias, 0, out, None)
        return lib.octree_nca_mx4_product(a, w, bias, 0, out, None)
    for x in (None, rows(G)):
        for bad in (dict(a=mx4(codes=None)), dict(w=mx4(9, 70, D, None)), dict(bias=G + 2),
                    dict(out=rows(None)), dict(out=rows(F + 2)), dict(out=rows(F, dtype=7)),
                    dict(out=rows(A + 16, cols=9)), dict(out=rows(B, cols=9)),
                    dict(out=rows(D, cols=9)), dict(out=rows(E, cols=9)),
                    dict(bias=F + 8), dict(bias=F - 32)):
            assert call(linear=x, **bad) == EINVAL, bad
        for bad in (dict(a=mx4(cols=71)), dict(w=mx4(9, 64, D, E)), dict(a=mx4(rows=-1)),
                    dict(w=mx4((1 << 20) + 1, 70, D, E)), dict(out=rows(F, stride=8))):
            assert call(linear=x, **bad) == ESHAPE, bad
        assert call(a=mx4(0, 70, None, None), out=rows(None), linear=x and rows(None)) == OK
    for bad in (rows(None), rows(G + 2), rows(A), rows(B), rows(F, cols=70), rows(G, dtype=5)):
        assert call(linear=bad) == EINVAL
    assert call(linear=rows(G, stride=69)) == ESHAPE
    # the inputs' codes are written: not over the weights or the bias
    assert call(linear=rows(G), w=mx4(9, 70, A + 256, E)) == EINVAL
    assert call(linear=rows(G), bias=B + 16) == EINVAL
    assert lib.octree_nca_mx4_product(None, mx4(), None, 0, rows(F), None) == EINVAL
    assert lib.octree_nca_mx4_linear(rows(G), None, mx4(), None, 0, rows(F), None) == EINVAL
    # no outputs: nothing to write
    assert call(w=mx4(0, 70, None, None), out=rows(None)) == OK


def test_backward_refusals(lib):
    need = lib.octree_nca_mx4_backward_workspace_bytes(20, 70, 9)
    work = G + (1 << 36)

    def call(g=None, a=None, w=None, gin=None, gw=F, gb=None, ws=work, size=need):
        return lib.octree_nca_mx4_backward(g or rows(G, cols=9), a or mx4(), w or mx4(9, 70, D, E),
                                           gin, gw, gb, ws, size, None)
    other = G + (1 << 35)
    for bad in (dict(g=rows(None)), dict(g=rows(G + 2, cols=9)), dict(g=rows(G, dtype=4)),
                dict(a=mx4(codes=None)), dict(w=mx4(9, 70, None, E)), dict(ws=None),
                dict(ws=work + 8), dict(gw=F + 2), dict(gb=other + 1),
                dict(gin=rows(other, dtype=F16)), dict(gin=rows(None)),
                dict(gin=rows(G)), dict(gin=rows(A)), dict(gin=rows(F)), dict(gin=rows(work)),
                dict(gw=G), dict(gw=B), dict(gw=E), dict(gw=work + 4), dict(gb=F + 4),
                dict(gb=work), dict(gb=D), dict(ws=A), dict(ws=G)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(w=mx4(9, 71, D, E)), dict(w=mx4(0, 70, None, None)), dict(a=mx4(rows=-2)),
                dict(g=rows(G, stride=8)), dict(gin=rows(other, stride=69)),
                dict(w=mx4((1 << 20) + 1, 70, D, E))):
        assert call(**bad) == ESHAPE, bad
    assert call(size=need - 1) == ESPACE
    assert lib.octree_nca_mx4_backward(rows(G), None, mx4(), None, F, None, work, need,
                                       None) == EINVAL


def test_dropout_refusals(lib):
    def call(d=None, x=None, gate=None, add=None, out=None, n=20, c=70):
        return lib.octree_nca_dropout(d or _Dropout(0.5, 1, 2, None), x or rows(A), gate, add,
                                      out or rows(B), n, c, None)
    nan = float("nan")
    for bad in (dict(d=_Dropout(-0.1, 0, 0, None)), dict(d=_Dropout(1.1, 0, 0, None)),
                dict(d=_Dropout(nan, 0, 0, None)), dict(d=_Dropout(0.5, 0, 0, E + 4)),
                dict(x=rows(None)), dict(x=rows(A + 2)), dict(x=rows(A, dtype=F16)),
                dict(x=rows(A, dtype=9)), dict(out=rows(B, dtype=BF16)), dict(out=rows(None)),
                dict(gate=rows(D, dtype=F16)), dict(add=rows(None)), dict(out=rows(A + 4)),
                dict(out=rows(A, stride=71)), dict(gate=rows(B - 4)), dict(add=rows(B + 280)),
                dict(d=_Dropout(0.5, 0, 0, B + 8))):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(n=-1), dict(c=-1), dict(n=1 << 40), dict(c=1 << 45, n=1),
                dict(x=rows(A, stride=69)), dict(gate=rows(D, stride=0)),
                dict(out=rows(B, stride=1 << 60))):
        assert call(**bad) == ESHAPE, bad
    assert call(n=0) == OK and call(c=0) == OK
    assert lib.octree_nca_dropout(None, rows(A), None, None, rows(B), 1, 1, None) == EINVAL
    assert lib.octree_nca_dropout(_Dropout(0.5, 0, 0, None), None, None, None, rows(B), 0, 1,
                                  None) == EINVAL


def test_shared_columns_of_one_buffer(lib):
    """Of two sets of columns of one buffer those that share a column overlap,
    however far apart their first elements are (apart: the GPU tests)."""
    def call(gin_at):
        return lib.octree_nca_mx4_backward(_Rows(G, 100, F32), mx4(), mx4(9, 70, D, E),
                                           _Rows(gin_at, 100, F32), None, None, None, 0, None)
    for at in (8, 31, -69, 99, 100 * 5 + 8, -100 * 5 - 1):
        assert call(G + 4 * at) == EINVAL, at


def test_binding_refuses(lib):
    """Checks of the binding that come before any GPU."""
    cpu = torch.zeros(4, 70)
    m = octnca.MX4Buffers(4, 70, *(torch.zeros(s, dtype=torch.uint8)
                                   for s in octnca.mx4_shapes(4, 70)))
    with pytest.raises(octnca.OctreeNCAError):
        m.struct()
    for bad in (cpu, torch.zeros(4, 70, dtype=torch.float64), cpu.t(), torch.zeros(())):
        with pytest.raises(octnca.OctreeNCAError):
            octnca._rows(bad, "x")
    with pytest.raises(TypeError):
        octnca._rows(cpu.numpy(), "x")
    with pytest.raises(octnca.OctreeNCAError):
        octnca.MX4Buffers(17, 70, *(torch.zeros(s, dtype=torch.uint8)
                                    for s in octnca.mx4_shapes(4, 70))).struct()


def test_header_example_of_the_layout():
    """Block b of row r begins at (((r / 16) * B + b) * 16 + r % 16) * 16."""
    rng = np.random.default_rng(3)
    values, codes, scales = cells4.quantise(rng.standard_normal((37, 70)))
    c, s = cells4.packed(codes, scales)
    flat_c, flat_s = c.reshape(-1), s.reshape(-1)
    for r, b in ((0, 0), (15, 2), (16, 1), (36, 2)):
        at = ((r // 16) * 3 + b) * 16 + r % 16
        assert flat_s[at] == scales[r, b]
        for k in range(32):
            assert flat_c[at * 16 + k // 2] >> (4 * (k % 2)) & 15 == codes[r, b, k]
    assert ctypes.sizeof(_MX4) == 32 and values.shape == (37, 70)
