"""The README's example of a head on a state: the text, and what it does."""
import os

import pytest
import torch

from conftest import ROOT
from head_example import EXAMPLE


def test_the_readme_has_it():
    path = os.path.join(ROOT, "README.md")
    if not os.path.exists(path):
        pytest.skip("sources without the README")
    with open(path) as f:
        assert "```python\n" + EXAMPLE + "```" in f.read()


@pytest.mark.gpu
def test_it_runs_and_its_gradients_train_it(gpu):
    from paper_2508_06993_amd.runtime import Parameters
    state = torch.randn(1, 30, 20, 16, device=gpu)
    names = {"torch": torch, "state": state}
    exec(EXAMPLE, names)
    layers = names["layers"]
    params = [t for layer in layers for t in (layer.weight, layer.bias)]
    grads = [t for layer in layers for t in (layer.grad_weight, layer.grad_bias)]
    before = [p.clone() for p in params]
    held = [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]
    Parameters(grads, params, *held).adamw(1e-2)
    for layer in layers:
        layer.refresh()
    # AdamW's first step goes by the gradients' signs: none is left out
    assert all((p != q).any() for p, q in zip(params, before))
    assert names["grad_state"].isfinite().all() and (names["grad_state"] != 0).any()
