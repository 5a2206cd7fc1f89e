"""Parameter lists of different lengths are refused, an empty gradient list beside
others too (no GPU: before an address is taken)."""
import pytest
import torch

import paper_2508_06993_amd as octnca


@pytest.mark.parametrize("name", ["params", "m", "v", "ema", "clipped"])
@pytest.mark.parametrize("grads,others", [(0, 1), (2, 1), (1, 2), (1, 0)])
def test_lists_of_different_lengths(name, grads, others):
    make = lambda n: [torch.zeros(3) for _ in range(n)]
    with pytest.raises(octnca.OctreeNCAError, match=f"{others} tensors for {grads} gradients"):
        octnca.param_structs(make(grads), **{name: make(others)})


def test_empty_lists():
    assert len(octnca.param_structs([], [], [], [])) == 1
