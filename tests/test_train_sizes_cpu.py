"""Tensors whose sizes do not fit a training call are refused before an address
of them is taken (no GPU: the tensors lie on the CPU, where a call whose sizes
fit is refused for that and nothing else)."""
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import Trainer

MODEL = octnca.Model(ndim=2, n_in=3)
STEPS, FACTORS = (2, 1), ((1, 2, 2),)


def weights(c=16, h=64, taps=9, levels=2):
    shapes = {"conv_w": (c, taps), "conv_b": (c,), "w1": (h, 2 * c), "b1": (h,), "w2": (c, h)}
    return [{k: torch.zeros(s) for k, s in shapes.items()} for _ in range(levels)]


def call(kept, **changed):
    a = dict(image=torch.zeros(1, 8, 12, 3), weights=weights(), target=torch.zeros(1, 8, 12, 2),
             grads=weights(), final_state=torch.zeros(1, 8, 12, 16))
    a.update(changed)
    step = octnca.octree_nca_train_step_kept if kept else octnca.octree_nca_train_step
    step(MODEL, a["image"], FACTORS, a["weights"], STEPS, 0.5, 0, a["target"],
         torch.zeros(1 << 20, dtype=torch.uint8), a["grads"], torch.zeros(1, dtype=torch.float64),
         a["final_state"])


@pytest.mark.parametrize("kept", [False, True])
def test_sizes_that_fit_get_as_far_as_the_device(library_path, kept):
    for ok in ({}, dict(final_state=None), dict(target=torch.zeros(96, 2))):
        with pytest.raises(octnca.OctreeNCAError, match="must be a device"):
            call(kept, **ok)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("name,bad", [
    ("target", lambda: torch.zeros(1, 8, 12, 1)),
    ("target", lambda: torch.zeros(1, 8, 11, 2)),
    ("image", lambda: torch.zeros(1, 8, 12, 1)),
    ("final_state", lambda: torch.zeros(1, 8, 12, 12)),
    ("weights", lambda: weights(12, 48)),
    ("weights", lambda: weights(taps=27)),
    ("weights", lambda: weights(levels=1)),
    ("weights", lambda: weights(levels=3)),
    ("grads", lambda: weights(12, 48)),
    ("grads", lambda: weights(levels=1)),
])
def test_sizes_that_do_not_fit(library_path, kept, name, bad):
    with pytest.raises(octnca.OctreeNCAError, match=f"^{name}"):
        call(kept, **{name: bad()})


@pytest.mark.parametrize("keep", [None, "i8"])
def test_trainer_refuses_weights_of_another_model(library_path, keep):
    for bad in (weights(12, 48), weights(20, 100), weights(taps=27), weights(levels=1),
                weights(levels=3)):
        with pytest.raises(octnca.OctreeNCAError, match="^weights"):
            Trainer(MODEL, (1, 8, 12), FACTORS, STEPS, bad, keep=keep)
