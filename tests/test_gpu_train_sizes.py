"""A Trainer with its buffers intact refuses images and targets of other sizes,
and goes on with right ones."""
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import Trainer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", [None, "i8"])
def test_trainer_refuses_other_sizes(gpu, keep):
    c, h, extent = 16, 64, (1, 8, 12)
    shapes = {"conv_w": (c, 9), "conv_b": (c,), "w1": (h, 2 * c), "b1": (h,), "w2": (c, h)}
    weights = [{k: torch.full(s, 0.01, device="cuda") for k, s in shapes.items()}]
    tr = Trainer(octnca.Model(ndim=2, n_in=3), extent, (), (2,), weights, keep=keep)
    image, target = torch.rand(extent + (3,), device="cuda"), torch.rand(extent + (2,), device="cuda")
    before = [w.clone() for w in weights[0].values()]
    for x, y, name in [(image, torch.rand(extent + (1,), device="cuda"), "target"),
                       (image[..., :1].contiguous(), target, "image"),
                       (image[:, :4].contiguous(), target[:, :4].contiguous(), "image"),
                       (image, target[:, :7].contiguous(), "target")]:
        with pytest.raises(octnca.OctreeNCAError, match=f"^{name}"):
            tr.step(x, y, 0.5, 0)
    assert int(tr.parameters.step) == 0
    assert all(torch.equal(a, b) for a, b in zip(before, weights[0].values()))
    tr.step(image, target, 0.5, 0)
    assert int(tr.parameters.step) == 1
