"""Writes in which a wave takes several blocks at a time, against the definition
and against writes of the same cells in pieces so small that it takes one.

Bounds: none between the two, the bits are the same; the definition's are those
of test_gpu_state_cache.py."""
import numpy as np
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import StateCache

from test_gpu_state_cache import HIDDEN, check_block

pytestmark = pytest.mark.gpu

# several blocks a wave from this many cells on; the cells of such a group
LINE = {"f32": 64 * 8192, "f16": 128 * 8192}
GROUP = {"f32": 64, "f16": 128}


def values(n, cells, c, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, 1, 1, cells, c), generator=gen, device="cuda")
    x *= torch.exp2(torch.linspace(-4, 7, c, device="cuda"))
    # each block of its own magnitude, so that no two share their scales
    x *= 1 + torch.arange(cells, device="cuda").div(32, rounding_mode="floor").remainder(
        7).float()[:, None]
    return x.to(torch.float32 if dtype == "f32" else torch.float16)


@pytest.mark.parametrize("c", [12, 16, 20])
@pytest.mark.parametrize("dtype,block", [("f32", 32), ("f16", 32), ("f16", 64)])
@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("tail", [0, 5, 32, 45, 64, 77, 96, 127])
def test_groups_equal_single_blocks(gpu, c, dtype, block, kind, tail):
    if tail >= GROUP[dtype]:
        pytest.skip("as a smaller tail")
    line = LINE[dtype]
    cells = line + tail
    model = octnca.Model(ndim=3, n_in=3, dtype=dtype, channels=c, hidden=HIDDEN[c])
    x = values(1, cells, c, dtype, 31 + tail)
    x[0, 0, 0, -1, 1] = float("nan")          # the last block, and one of a full group
    x[0, 0, 0, line // 2 + 40, 2] = float("-inf")
    grouped, single = (StateCache(model, (1, 1, cells), 2, kind, block) for _ in range(2))
    for cache in (grouped, single):
        cache.buffers.codes.fill_(77)
        cache.buffers.scales.fill_(-1)
    grouped.write(x, first=1)
    piece = line // 2
    for lo in range(0, cells, piece):
        single.write(x[:, :, :, lo:lo + piece].contiguous(), first=1, from_cell=lo)
    assert torch.equal(grouped.buffers.codes, single.buffers.codes)
    assert torch.equal(grouped.buffers.scales, single.buffers.scales)
    assert bool((grouped.buffers.codes[0] == 77).all()) and \
        bool((grouped.buffers.scales[0] == -1).all())
    back = grouped.read(torch.empty_like(x), first=1)
    blocks = -(-cells // block)
    for j in sorted({0, 1, 2, 3, line // 2 // block, line // 2 // block + 1, blocks - 6, blocks - 5,
                     blocks - 4, blocks - 3, blocks - 2, blocks - 1}):
        at = slice(j * block, min(cells, (j + 1) * block))
        cut = lambda t: t[0, 0, 0, at].cpu().numpy()
        check_block(cut(x), grouped.buffers.codes[1, at].cpu().numpy(),
                    grouped.buffers.scales[1, j].cpu().numpy(), cut(back), kind, dtype)


@pytest.mark.parametrize("dtype,block", [("f32", 32), ("f16", 32), ("f16", 64)])
def test_groups_of_many_states(gpu, dtype, block):
    """Many states that pass the line together, each with a partial last group and
    a slot of its own; some given twice, some outside."""
    model = octnca.Model(ndim=3, n_in=3, dtype=dtype, channels=16, hidden=64)
    cells = 5 * GROUP[dtype] + 37
    n = LINE[dtype] // cells + 9
    x = values(n, cells, 16, dtype, 41)
    order = np.random.default_rng(5).permutation(n + 20)[:n]
    order[3], order[5], order[8] = order[n - 1], -1, n + 20
    cache, alone = (StateCache(model, (1, 1, cells), n + 20, "i8", block) for _ in range(2))
    slots = torch.from_numpy(order).cuda()
    cache.write(x, slots)
    for i in range(0, n, 97):     # a few of them below the line
        alone.write(x[i:i + 97], slots[i:i + 97].contiguous())
    assert torch.equal(cache.buffers.codes, alone.buffers.codes)
    assert torch.equal(cache.buffers.scales, alone.buffers.scales)
