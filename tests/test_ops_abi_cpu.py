"""Refusals of the state-cache, parameter-list and kept-training entry points
without a GPU: every call below fails validation, so no HIP call is made."""
import ctypes
import math

import numpy as np
import pytest

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import (_AdamW, _Extent, _Keep, _LevelGrads, _LevelWeights, _Model,
                                  _Param, _ParamList, _StateCache)
from quantise import e4m3_round, e4m3_values, read_back

OK, EINVAL, EUNSUP, ESHAPE, ESPACE = 0, -1, -2, -3, -5
A, B, D, E = 0x7f0000001000, 0x7f1000000000, 0x7f2000000000, 0x7f3000000000   # never dereferenced


@pytest.fixture(scope="module")
def lib(library_path):
    return octnca.lib()


def cache_call(lib, write=True, m=None, states=A, start=0, count=64, n=1, slots=None, first=0,
               **cache):
    c = dict(code=0, block=64, slots=2, cells=100, codes=B, scales=D)
    c.update(cache)
    fn = lib.octree_nca_state_cache_write if write else lib.octree_nca_state_cache_read
    return fn(ctypes.byref(m or _Model(2, 16, 64, 3, 0)), ctypes.byref(_StateCache(**c)), states,
              start, count, n, slots, first, None)


@pytest.mark.parametrize("write", [True, False])
def test_cache_refusals(lib, write):
    call = lambda **k: cache_call(lib, write, **k)
    for bad in (dict(states=None), dict(codes=None), dict(scales=None), dict(code=2),
                dict(code=-1), dict(block=48), dict(block=0), dict(start=1), dict(n=-1),
                dict(count=-1), dict(start=-64), dict(states=A + 4), dict(codes=B + 1),
                dict(scales=D + 4), dict(slots=E + 4), dict(states=B), dict(states=D + 64),
                dict(slots=A)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(cells=0), dict(cells=-5), dict(count=101),
                dict(start=64, count=37), dict(start=128), dict(first=2), dict(first=-1),
                dict(n=3), dict(first=1, n=2), dict(cells=1 << 40)):
        assert call(**bad) == ESHAPE, bad
    assert call(m=_Model(2, 16, 63, 3, 0)) == EUNSUP
    assert call(m=_Model(2, 16, 64, 3, octnca.OCTNCA_BF16)) == EUNSUP
    # nothing to do
    assert call(n=0) == OK and call(count=0) == OK and call(n=0, states=None) == OK


def test_cache_slot_counts(lib):
    bad = _StateCache(0, 64, -1, 100, B, D)
    m = _Model(2, 16, 64, 3, 0)
    assert lib.octree_nca_state_cache_write(ctypes.byref(m), ctypes.byref(bad), A, 0, 64, 1, None,
                                            0, None) == ESHAPE
    huge = _StateCache(0, 64, 1 << 62, 100, B, D)
    assert lib.octree_nca_state_cache_write(ctypes.byref(m), ctypes.byref(huge), A, 0, 64, 1, None,
                                            0, None) == ESHAPE
    assert lib.octree_nca_state_cache_write(ctypes.byref(m), None, A, 0, 64, 1, None, 0,
                                            None) == EINVAL
    assert lib.octree_nca_state_cache_write(None, ctypes.byref(bad), A, 0, 64, 1, None, 0,
                                            None) == EINVAL


def test_a_write_ends_at_a_block_or_the_state(lib):
    assert cache_call(lib, True, count=63) == EINVAL
    assert cache_call(lib, True, start=64, count=20) == EINVAL


def params(*items):
    base = dict(count=10, grad=A, clipped=None, param=None, m=None, v=None, ema=None, grad_dtype=0,
                clipped_dtype=0)
    return (_Param * max(1, len(items)))(*[_Param(**{**base, **k}) for k in items]), len(items)


FULL = dict(param=B, m=D, v=E)


def test_param_list_refusals(lib):
    def both(items, want):
        arr, n = params(*items)
        assert lib.octree_nca_param_table_bytes(arr, n) == 0
        out = _ParamList()
        assert lib.octree_nca_param_table(arr, n, 0x7f9000000000, 1 << 30, ctypes.byref(out),
                                          None) == want
    both([dict(grad=None)], EINVAL)
    both([dict(count=-1)], ESHAPE)
    both([dict(count=1 << 40)], ESHAPE)
    both([dict(grad_dtype=3)], EINVAL)
    both([dict(grad=A + 2)], EINVAL)
    both([dict(grad_dtype=2, grad=A + 1)], EINVAL)
    both([dict(clipped=B, clipped_dtype=9)], EINVAL)
    both([dict(clipped=B + 2)], EINVAL)
    both([dict(param=B)], EINVAL)
    both([dict(param=B, m=D)], EINVAL)
    both([dict(ema=B)], EINVAL)
    both([dict(FULL, m=D + 1)], EINVAL)
    both([dict(clipped=B), dict(grad=A + 64)], EINVAL)            # given for one only
    both([FULL, dict(grad=A + 64)], EINVAL)
    arr, n = params(dict())
    out = ctypes.byref(_ParamList())
    assert lib.octree_nca_param_table_bytes(None, 1) == 0
    assert lib.octree_nca_param_table_bytes(arr, -1) == 0
    need = lib.octree_nca_param_table_bytes(arr, n)
    assert need > 0
    assert lib.octree_nca_param_table(arr, n, None, need, out, None) == EINVAL
    assert lib.octree_nca_param_table(arr, n, B, need, None, None) == EINVAL
    assert lib.octree_nca_param_table(arr, n, B + 8, need, out, None) == EINVAL
    assert lib.octree_nca_param_table(arr, n, B, need - 1, out, None) == ESPACE
    assert lib.octree_nca_param_table(arr, n, A, need, out, None) == EINVAL   # over a gradient


@pytest.mark.parametrize("items", [
    [dict(clipped=A + 4)],                                   # part of the gradient
    [dict(clipped=A, clipped_dtype=1)],                      # the gradient in another type
    [dict(FULL, m=B + 36)],
    [dict(FULL), dict(param=B + 4096, m=D + 8, v=E + 4096, grad=A + 4096)],
    [dict(clipped=B), dict(grad=B + 16, clipped=D)],         # a gradient that another tensor writes
    [dict(clipped=B), dict(grad=A + 512, clipped=B + 36)],
])
def test_param_list_overlaps(lib, items):
    arr, n = params(*items)
    need = lib.octree_nca_param_table_bytes(arr, n)
    assert need > 0
    assert lib.octree_nca_param_table(arr, n, 0x7f9000000000, need, ctypes.byref(_ParamList()),
                                      None) == EINVAL


def test_table_bytes_grow_with_chunks(lib):
    size = lambda n: lib.octree_nca_param_table_bytes(*params(dict(count=n)))
    assert size(1) == size(4096) < size(4097) == size(8192) < size(1 << 20)
    # a tensor that starts inside a group of four may need one chunk more
    off = lib.octree_nca_param_table_bytes(*params(dict(count=4096, grad=A + 4)))
    assert off == size(4097)
    assert lib.octree_nca_param_table_bytes(*params()) == \
        lib.octree_nca_param_table_bytes(*params(dict(count=0, grad=None)))


def plist(has):
    return ctypes.byref(_ParamList(A, 1, 10, 40, has))


def test_gradient_calls_refuse(lib):
    nan, inf = float("nan"), float("inf")
    norm, clip = lib.octree_nca_grad_norm, lib.octree_nca_clip_grads
    assert norm(None, 1.0, B, None) == EINVAL
    assert norm(plist(0), 1.0, None, None) == EINVAL
    assert norm(ctypes.byref(_ParamList()), 1.0, B, None) == EINVAL
    for s in (0.0, -1.0, nan, inf):
        assert norm(plist(0), s, B, None) == EINVAL
        assert clip(plist(1), s, 1.0, B, None) == EINVAL
    for m in (0.0, -1.0, nan):
        assert clip(plist(1), 1.0, m, B, None) == EINVAL
    assert clip(plist(2), 1.0, 1.0, B, None) == EINVAL         # no `clipped`
    assert norm(plist(0), 1.0, B + 2, None) == EINVAL


def test_adamw_refuses(lib):
    good = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, max_norm=1.0, scale=1.0,
                ema_decay=0.9)
    nan, inf = float("nan"), float("inf")

    def call(l=None, step=B, norm=None, h=None, **k):
        h = ctypes.byref(_AdamW(**{**good, **k})) if h is None else h
        return lib.octree_nca_adamw(l if l is not None else plist(2), h, step, norm, None)
    for bad in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1),
                dict(beta2=nan), dict(beta2=1.0), dict(eps=0.0), dict(eps=1e-60), dict(eps=nan),
                dict(weight_decay=-0.1), dict(weight_decay=inf), dict(max_norm=0.0),
                dict(max_norm=nan), dict(scale=0.0), dict(scale=inf), dict(ema_decay=1.1),
                dict(ema_decay=nan), dict(step=None), dict(step=B + 4), dict(norm=D + 2),
                dict(l=plist(1)), dict(l=plist(0))):
        assert call(**bad) == EINVAL, bad
    assert lib.octree_nca_adamw(plist(2), None, B, None, None) == EINVAL
    assert lib.octree_nca_adamw(None, ctypes.byref(_AdamW(**good)), B, None, None) == EINVAL


def test_kept_training_refuses(lib):
    m = ctypes.byref(_Model(2, 16, 64, 3, 0))
    steps, f = (ctypes.c_int32 * 2)(3, 2), (ctypes.c_int32 * 3)(1, 2, 2)
    e = _Extent(1, 8, 8)
    size = lib.octree_nca_train_kept_workspace_bytes
    good = ctypes.byref(_Keep(0, 64))
    need = size(m, e, 2, f, steps, good)
    assert 0 < need < lib.octree_nca_train_workspace_bytes(m, e, 2, f, (ctypes.c_int32 * 2)(40, 40))
    for k in (_Keep(2, 64), _Keep(-1, 64), _Keep(0, 16), _Keep(0, 0)):
        assert size(m, e, 2, f, steps, ctypes.byref(k)) == 0
    assert size(m, e, 2, f, steps, None) == 0
    assert size(m, _Extent(1, 7, 8), 2, f, steps, good) == 0
    assert size(ctypes.byref(_Model(2, 16, 64, 3, 1)), e, 2, f, steps, good) == 0
    big = _Extent(1, 1 << 18, 1 << 18)       # 2^36 cells, 2^31 - 1 steps: more than 2^64 bytes
    assert size(m, big, 1, f, (ctypes.c_int32 * 1)(2 ** 31 - 1), good) == 0
    ws = (_LevelWeights * 2)(*[_LevelWeights(A, A, A, A, A)] * 2)
    gs = (_LevelGrads * 2)(*[_LevelGrads(A, A, A, A, A)] * 2)
    step = lib.octree_nca_train_step_kept

    def call(image=A, rate=0.5, target=B, keep=good, work=D, nbytes=need, grads=gs, loss=E,
             final=None):
        return step(m, image, e, 2, f, ws, steps, rate, 0, target, keep, work, nbytes, grads, loss,
                    final, None)
    for bad in (dict(image=None), dict(target=None), dict(work=None), dict(loss=None),
                dict(grads=None), dict(rate=1.5), dict(rate=math.nan), dict(keep=None),
                dict(keep=ctypes.byref(_Keep(0, 31))), dict(work=D + 8), dict(image=D + 256),
                dict(target=D), dict(final=D + 512),
                dict(grads=(_LevelGrads * 2)(_LevelGrads(A, A, A, A, A)))):
        assert call(**bad) == EINVAL, bad
    assert call(nbytes=need - 1) == ESPACE


def test_e4m3_of_the_tests_is_torch_s():
    """The tests' own table and rounding against torch's type."""
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(e4m3_values(), want, equal_nan=True)
    x = np.random.default_rng(1).uniform(-448, 448, 20000).astype(np.float32)
    x *= np.exp2(np.random.default_rng(2).integers(-12, 1, 20000)).astype(np.float32)
    got = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(e4m3_round(x.astype(np.float64)), got.astype(np.float64))


@pytest.mark.parametrize("code,bound", [("i8", 1 / 254), ("f8", 1 / 16)])
def test_read_back_error(code, bound):
    """The definition's error: half a step of the block's largest value (I8), or
    half a unit of the value's three mantissa bits, 2^-4 of it (F8, above its
    subnormals)."""
    x = np.random.default_rng(3).normal(0, 1, (1, 5, 40, 16))
    y = read_back(x, code, 32)
    if code == "i8":
        for i in range(0, 200, 32):
            b, r = x.reshape(-1, 16)[i:i + 32], y.reshape(-1, 16)[i:i + 32]
            assert np.all(np.abs(b - r) <= np.abs(b).max(0) * bound * (1 + 1e-12))
    else:
        top = np.abs(x).max()
        big = np.abs(x) > top * 2.0 ** -13
        assert np.all(np.abs(x - y)[big] <= np.abs(x)[big] * bound)
