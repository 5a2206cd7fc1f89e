"""Objects made on one stream and used at once on another: the fills of their own
buffers come before the use, however far behind the making stream is."""
import contextlib

import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import Parameters, StateCache, Trainer

pytestmark = pytest.mark.gpu

COUNTS = [3000, 17, 40_001]           # two launches a call
SMALL = [300, 17, 1000]               # one


def keep_busy():
    """Some tens of milliseconds of work on the current stream, and memory of many
    sizes that it still reads when the allocator hands it out again."""
    a = torch.randn(4096, 4096, device="cuda") / 64
    junk = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
            for n in (4, 8, 512, 1 << 13, 1 << 15, 1 << 17, 1 << 21)]
    for _ in range(30):
        a = a @ a / 64
    return [j + 1 for j in junk]


def lists(counts, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda: [torch.randn(n, generator=gen, device="cuda") for n in counts]
    return make(), make(), make(), [x.square() for x in make()]


def other_stream(kind):
    """(context of the call, its stream argument, the stream to wait for)"""
    side = torch.cuda.Stream()
    if kind == "current":
        return torch.cuda.stream(side), None, side
    return contextlib.nullcontext(), side if kind == "object" else side.cuda_stream, side


@pytest.mark.parametrize("kind", ["object", "handle", "current"])
@pytest.mark.parametrize("made_on_it", [False, True])
@pytest.mark.parametrize("counts", [COUNTS, SMALL], ids=["two-launches", "one-launch"])
def test_a_list_used_at_once(gpu, kind, made_on_it, counts):
    want = lists(counts)
    norm = float(Parameters(*want).adamw(0.01, max_norm=1.0))
    got = lists(counts)
    context, stream, side = other_stream(kind)
    torch.cuda.synchronize()
    keep_busy()
    if made_on_it and stream is not None:
        p = Parameters(*got, stream=stream)
    else:
        p = Parameters(*got)
    with context:
        returned = p.adamw(0.01, max_norm=1.0, stream=stream)
    torch.cuda.synchronize()
    assert int(p.step) == 1 and float(returned) == norm
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("kind", ["object", "handle", "current"])
def test_a_cache_used_at_once(gpu, kind):
    model = octnca.Model(ndim=2, n_in=3)
    x = torch.randn((2, 1, 64, 64, 16), device="cuda")
    want = StateCache(model, (1, 64, 64), 2)
    want.write(x)
    back = torch.empty_like(x)
    context, stream, side = other_stream(kind)
    torch.cuda.synchronize()
    keep_busy()
    cache = StateCache(model, (1, 64, 64), 2)
    with context:
        cache.write(x, stream=stream)
        cache.read(back, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(cache.buffers.codes, want.buffers.codes)
    assert torch.equal(cache.buffers.scales, want.buffers.scales)
    assert torch.equal(back, want.read(torch.empty_like(x)))


@pytest.mark.parametrize("keep", [None, "i8"])
@pytest.mark.parametrize("kind", ["object", "handle", "current"])
def test_a_trainer_used_at_once(gpu, keep, kind):
    extent, c, h = (1, 16, 24), 16, 64
    shapes = {"conv_w": (c, 9), "conv_b": (c,), "w1": (h, 2 * c), "b1": (h,), "w2": (c, h)}
    gen = torch.Generator(device="cuda").manual_seed(2)
    start = [{k: torch.randn(s, generator=gen, device="cuda") * 0.1 for k, s in shapes.items()}
             for _ in range(2)]
    image = torch.rand(extent + (3,), generator=gen, device="cuda")
    target = torch.rand(extent + (2,), generator=gen, device="cuda")
    results = []
    for at_once in (False, True):
        weights = [{k: v.clone() for k, v in w.items()} for w in start]
        context, stream, side = (other_stream(kind) if at_once else
                                 (contextlib.nullcontext(), None, None))
        torch.cuda.synchronize()
        if at_once:
            keep_busy()
        tr = Trainer(octnca.Model(ndim=2, n_in=3), extent, ((1, 2, 2),), (3, 2), weights, keep=keep,
                     max_norm=1.0)
        with context:
            for k in range(2):
                tr.step(image, target, 0.5, k, stream=stream)
        torch.cuda.synchronize()
        assert int(tr.parameters.step) == 2
        results.append([t for sets in (weights, tr.ema) for w in sets for t in w.values()] +
                       [tr.loss])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_memory_of_a_list_that_is_gone(gpu):
    """A list given up while its calls are still to run: its table is not handed
    out before they are through."""
    want = lists(SMALL)
    Parameters(*want).adamw(0.01, max_norm=1.0)
    got = lists(SMALL)
    side = torch.cuda.Stream()
    p = Parameters(*got)
    torch.cuda.synchronize()
    at, size = p.table.data_ptr(), p.table.numel()
    with torch.cuda.stream(side):
        keep_busy()
        p.adamw(0.01, max_norm=1.0)
    del p
    new = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert not side.query()
    assert all(t.data_ptr() + size <= at or at + size <= t.data_ptr() for t in new)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("made_on_it", [False, True])
def test_the_default_stream_by_its_handle(gpu, made_on_it):
    """Handle 0 is the default stream, also where another one is current."""
    want = lists(COUNTS)
    Parameters(*want).adamw(0.01, max_norm=1.0)
    got = lists(COUNTS)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        keep_busy()
        p = Parameters(*got, stream=0) if made_on_it else Parameters(*got)
        p.adamw(0.01, max_norm=1.0, stream=0)
        if made_on_it:      # nothing here has waited for the busy stream
            torch.cuda.default_stream().synchronize()
            assert not side.query()
    torch.cuda.synchronize()
    assert int(p.step) == 1
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
