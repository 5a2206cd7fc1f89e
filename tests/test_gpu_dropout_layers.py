"""Masks of several layers over several steps: of one seed and index + step there is one
mask, so layers take seeds of their own."""
import pytest
import torch

from paper_2508_06993_amd.runtime import Dropout

pytestmark = pytest.mark.gpu


def masks(drops, step, steps, index):
    """Which of 4096 elements each layer drops at each step."""
    x = torch.ones(64, 64, device="cuda")
    out = {}
    for t in range(steps):
        step.fill_(t)
        for k, drop in enumerate(drops):
            out[k, t] = drop(x, torch.empty_like(x), index=index[k]) == 0
    return out


def test_seeds_of_their_own(gpu):
    """No two of sixteen masks are alike: each pair differs in about half of the elements
    (5 sigma of 4096 draws of rate 1/2)."""
    step = torch.zeros(1, dtype=torch.int64, device=gpu)
    all_masks = list(masks([Dropout(0.5, 40 + k, step) for k in range(4)], step, 4,
                           [0] * 4).values())
    for i, a in enumerate(all_masks):
        for b in all_masks[:i]:
            assert abs((a != b).sum().item() - 2048) < 5 * 32


def test_one_seed(gpu):
    step = torch.zeros(1, dtype=torch.int64, device=gpu)
    near = masks([Dropout(0.5, 40, step) for _ in range(2)], step, 3, [0, 1])
    assert torch.equal(near[1, 0], near[0, 1]) and torch.equal(near[1, 1], near[0, 2])
    far = list(masks([Dropout(0.5, 40, step) for _ in range(2)], step, 3, [0, 1 << 40]).values())
    assert not any(torch.equal(a, b) for i, a in enumerate(far) for b in far[:i])
