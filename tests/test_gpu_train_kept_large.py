"""The kept training step at the sizes it is for: levels whose backward takes the
large tiles, whose codes are streamed past the last-level cache, and with more
windows than one.

The forward is octree_nca_train_step's: the same bits of loss and final state.
The gradients are compared with those of the states that read back from a cache
of their own, one octree_nca_step_backward a step and octree_nca_upsample_backward
between levels.  Both sides are fp32 at the same states, so they differ in the
order of sums: a state gradient by 2e-5 of the largest a step (the bound of one
step against the oracle), carried through t steps by about sqrt(t) of that, a
weight gradient by 1e-4 more; at most 100 steps here: 3e-4, taken as 1e-3."""
import numpy as np
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import StateCache, upload_weights

from parity import max_rel_err, to_np
from test_gpu_train_kept import KEYS, TOL_TRAIN, dev, make

pytestmark = pytest.mark.gpu

SEED, RATE = 3, 0.5
PATCH = (320, 320)
CASES = [
    ("patch", 2, 3, (1,) + PATCH, ((1, 2, 2),) * 4, (20,) * 5, 16, 64),
    ("streamed", 2, 3, (1, 1000, 1100), (), (5,), 16, 64),
    ("ragged-tiles", 2, 1, (1, 626, 354), ((1, 2, 2),), (7, 9), 16, 64),
    ("volume", 3, 1, (12, 96, 96), ((2, 2, 2),), (6, 10), 16, 64),
    ("patch-12", 2, 3, (1,) + PATCH, ((1, 2, 2),), (9, 6), 12, 48),
    ("volume-20", 3, 3, (6, 60, 62), ((1, 2, 2),), (5, 6), 20, 100),
]


def train(model, image, target, up, factors, steps, c, keep):
    """(loss, final state, gradients) of one training step."""
    extent = image.shape[:3]
    grads = [{k: torch.full_like(w[k], 7.0) for k in KEYS} for w in up]
    loss = torch.zeros(1, dtype=torch.float64, device="cuda")
    final = torch.empty(tuple(extent) + (c,), device="cuda")
    size = (octnca.octree_nca_train_kept_workspace_bytes if keep else
            octnca.octree_nca_train_workspace_bytes)
    work = torch.empty(size(model, extent, factors, steps, *keep), dtype=torch.uint8, device="cuda")
    step = octnca.octree_nca_train_step_kept if keep else octnca.octree_nca_train_step
    step(model, image, factors, up, steps, RATE, SEED, target, work, grads, loss, final, *keep)
    return loss, final, grads


def level_states(model, first, weights, lvl, steps):
    """The state before each step and after the last, of runs with one step a launch."""
    states = [first]
    for n in range(1, steps + 1):
        b = [first.clone(), torch.empty_like(first)]
        states.append(b[octnca.octree_nca_run_level(model, *b, weights, lvl, n, RATE, SEED)])
    return states


def reference(ndim, n_in, image, target, up, factors, steps, c, h, code, block):
    """(final state, gradients) step by step, the backward at states read back."""
    model = octnca.Model(ndim=ndim, n_in=n_in, channels=c, hidden=h)
    runs = octnca.Model(ndim=ndim, n_in=n_in, channels=c, hidden=h,
                        kernel="mfma_bf16x3,mfma_1step" if c == 16 else "valu")
    images = [image]
    for f in factors:
        shape = tuple(n // k for n, k in zip(images[-1].shape[:3], f))
        images.append(torch.empty(shape + (n_in,), device="cuda"))
    octnca.octree_nca_build_pyramid(runs, image, factors, images[1:])
    back, state = [None] * len(steps), None
    for lvl in range(len(steps) - 1, -1, -1):
        extent = tuple(images[lvl].shape[:3])
        first = torch.zeros(extent + (c,), device="cuda")
        if state is None:
            first[..., :n_in] = images[lvl]
        else:
            octnca.octree_nca_upsample(runs, state, factors[lvl], images[lvl], first)
        states = level_states(runs, first, up[lvl], lvl, steps[lvl])
        state = states.pop()
        back[lvl] = torch.stack(states)
        cache = StateCache(model, extent, len(states), code, block)
        cache.write(back[lvl])
        cache.read(back[lvl])
    g, loss = torch.empty_like(state), torch.zeros(1, dtype=torch.float64, device="cuda")
    work = torch.empty(octnca.octree_nca_readout_mse_workspace_bytes(image.shape[:3]),
                       dtype=torch.uint8, device="cuda")
    octnca.octree_nca_readout_mse(model, state, target, g, loss, work)
    grads = [{k: torch.zeros_like(w[k]) for k in KEYS} for w in up]
    for lvl in range(len(steps)):
        extent = tuple(images[lvl].shape[:3])
        work = torch.empty(octnca.octree_nca_step_backward_workspace_bytes(model, extent),
                           dtype=torch.uint8, device="cuda")
        for t in range(steps[lvl] - 1, -1, -1):
            octnca.octree_nca_step_backward(model, back[lvl][t], g, up[lvl], lvl, t, RATE, SEED, g,
                                            grads[lvl], work)
        if lvl + 1 < len(steps):
            coarse = torch.empty(tuple(images[lvl + 1].shape[:3]) + (c,), device="cuda")
            octnca.octree_nca_upsample_backward(model, g, factors[lvl], coarse)
            g = coarse
    return state, grads


@pytest.mark.parametrize("code,block", [("i8", 64), ("f8", 32)])
@pytest.mark.parametrize("name,ndim,n_in,extent,factors,steps,c,h", CASES,
                         ids=[c[0] for c in CASES])
def test_kept_step_at_full_size(gpu, name, ndim, n_in, extent, factors, steps, c, h, code, block):
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h, seed=23)
    for w in weights:     # states stay near the image's through 100 steps
        for k in KEYS:
            getattr(w, k)[...] *= 0.3
    image, target, up = dev(image), dev(target), upload_weights(weights)
    model = octnca.Model(ndim=ndim, n_in=n_in, channels=c, hidden=h)
    loss, final, grads = train(model, image, target, up, factors, steps, c, (code, block))
    whole_loss, whole_final, whole = train(model, image, target, up, factors, steps, c, ())
    assert torch.equal(final, whole_final) and torch.equal(loss, whole_loss)
    state, want = reference(ndim, n_in, image, target, up, factors, steps, c, h, code, block)
    assert torch.equal(state, final)
    for lvl in range(len(steps)):
        for k in KEYS:
            err = max_rel_err(to_np(grads[lvl][k]), to_np(want[lvl][k]))
            assert np.isfinite(err) and err <= TOL_TRAIN, (lvl, k, err)
