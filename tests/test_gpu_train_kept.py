"""The training step with its states kept in 8 bits, and training with updates.

The oracle of the kept step is the fp64 backward over a tape whose states went
through the cache's definition (quantise.py).  These states are the GPU's, from
level runs of the training forward's arithmetic: the oracle's own differ in their
last bits, and one value that lies at a tie between two codes then moves a small
case's gradient by more than all arithmetic does.  Bounds: the forward's loss and
final state as in the other training step's tests (TOL_TRAIN, the split-bf16
rounding); the gradients, at the same states, by fp32 products and sums
(TOL_TRAIN covers whole steps there too).  Along the gradient the loss's
difference quotient is |grad|^2 up to the gradient's own error: at most 0.5% (I8)
and 1.1% (F8) in 2-norm for these cases by the oracle, doubled here."""
import numpy as np
import pytest
import torch

import oracle
import paper_2508_06993_amd as octnca
from paper_2508_06993_amd.runtime import Trainer, upload_weights
from synthetic import LevelWeights

from parity import max_rel_err, to_np
from quantise import read_back

pytestmark = pytest.mark.gpu

KEYS = ("conv_w", "conv_b", "w1", "b1", "w2")
TOL_TRAIN = 1e-3
SLOPE = {"i8": 0.01, "f8": 0.022}

CASES = [
    ("2d", 2, 3, (1, 24, 40), ((1, 2, 2), (1, 2, 2)), (7, 5, 6), 16, 64),
    ("2d-zero", 2, 3, (1, 36, 68), ((1, 2, 2), (1, 3, 2)), (4, 0, 3), 16, 64),
    ("2d-none-at-the-finest", 2, 1, (1, 20, 36), ((1, 2, 2),), (0, 9), 16, 64),
    ("2d-one", 2, 3, (1, 33, 61), (), (1,), 16, 64),
    ("2d-long", 2, 3, (1, 9, 13), (), (41,), 16, 64),
    ("3d", 3, 1, (4, 12, 16), ((1, 2, 2),), (5, 4), 16, 64),
    ("2d-12", 2, 3, (1, 22, 30), ((1, 2, 2),), (6, 5), 12, 48),
    ("3d-20", 3, 3, (2, 10, 14), ((1, 2, 2),), (5, 3), 20, 100),
]


def make(ndim, n_in, extent, factors, steps, c, h, seed=5):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.normal(0, 0.1, s).astype(np.float32)
    image = rng.uniform(0, 1, extent + (n_in,)).astype(np.float32)
    target = rng.uniform(0, 1, extent + (2,)).astype(np.float32)
    weights = [LevelWeights(conv_w=f(c, 3 ** ndim), conv_b=f(c), w1=f(h, 2 * c), b1=f(h), w2=f(c, h))
               for _ in steps]
    return image, target, weights


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def kept(model, image, target, weights, factors, steps, code, block, c):
    """(loss, final state, gradients) of octree_nca_train_step_kept."""
    extent = image.shape[:3]
    up = upload_weights(weights)
    grads = [{k: torch.full_like(w[k], 7.0) for k in KEYS} for w in up]     # overwritten
    loss = torch.zeros(1, dtype=torch.float64, device="cuda")
    final = torch.empty(extent + (c,), dtype=torch.float32, device="cuda")
    n = octnca.octree_nca_train_kept_workspace_bytes(model, extent, factors, steps, code, block)
    work = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")    # NaN wherever not written
    octnca.octree_nca_train_step_kept(model, dev(image), factors, up, steps, 0.5, 3, dev(target),
                                      work[:n], grads, loss, final, code, block)
    torch.cuda.synchronize()
    assert bool((work[n:] == 0xFF).all())
    return float(loss), to_np(final), [{k: to_np(v) for k, v in g.items()} for g in grads]


def gpu_states(ndim, n_in, c, h, image, weights, factors, steps):
    """Per level the states before each step and after the last, of level runs
    with one step per launch."""
    kernel = "mfma_bf16x3,mfma_1step" if c == 16 else "valu"
    model = octnca.Model(ndim=ndim, n_in=n_in, channels=c, hidden=h, kernel=kernel)
    up = upload_weights(weights)
    images = [dev(image)]
    for f in factors:
        shape = tuple(n // k for n, k in zip(images[-1].shape[:3], f))
        images.append(torch.empty(shape + (n_in,), device="cuda"))
    octnca.octree_nca_build_pyramid(model, images[0], factors, images[1:])
    out, state = [None] * len(steps), None
    for lvl in range(len(steps) - 1, -1, -1):
        first = torch.zeros(images[lvl].shape[:3] + (c,), device="cuda")
        if state is None:
            first[..., :n_in] = images[lvl]
        else:
            octnca.octree_nca_upsample(model, state, factors[lvl], images[lvl], first)
        states = [first]
        for n in range(1, steps[lvl] + 1):
            b = [first.clone(), torch.empty_like(first)]
            states.append(b[octnca.octree_nca_run_level(model, *b, up[lvl], lvl, n, 0.5, 3)])
        out[lvl], state = [to_np(s) for s in states], states[-1]
    return out


@pytest.mark.parametrize("code,block", [("i8", 64), ("f8", 32), ("i8", 128)])
@pytest.mark.parametrize("name,ndim,n_in,extent,factors,steps,c,h", CASES,
                         ids=[c[0] for c in CASES])
def test_kept_step_matches_oracle(gpu, name, ndim, n_in, extent, factors, steps, c, h, code, block):
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h)
    model = octnca.Model(ndim=ndim, n_in=n_in, channels=c, hidden=h)
    loss, final, grads = kept(model, image, target, weights, factors, steps, code, block, c)
    kw = dict(ndim=ndim, n_in=n_in, factors=factors, seed=3, fire_rate=0.5)
    tape = oracle.train_forward(image, weights, channels=c, steps=steps, dtype=np.float32, **kw)
    want_loss, _ = oracle.readout_mse(tape.final, target)
    assert loss == pytest.approx(want_loss, rel=TOL_TRAIN)
    assert max_rel_err(final, tape.final) <= TOL_TRAIN
    states = gpu_states(ndim, n_in, c, h, image, weights, factors, steps)
    assert np.array_equal(states[0][-1], final)
    stored = type(tape)([[read_back(s, code, block).astype(np.float32) for s in st[:-1]] + [st[-1]]
                         for st in states])
    _, g_final = oracle.readout_mse(final, target)
    want = oracle.train_backward(stored, weights, g_final=g_final, **kw)
    for lvl in range(len(steps)):
        for k in KEYS:
            if steps[lvl] == 0:
                assert not grads[lvl][k].any()
                continue
            err = max_rel_err(grads[lvl][k], getattr(want[lvl], k))
            assert err <= TOL_TRAIN, (lvl, k, err)


@pytest.mark.parametrize("code", ["i8", "f8"])
def test_kept_gradient_against_differences(gpu, code):
    """The loss's slope along the kept gradient, by differences of the oracle's
    float64 loss."""
    _, ndim, n_in, extent, factors, steps, c, h = CASES[0]
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h)
    model = octnca.Model(ndim=ndim, n_in=n_in)
    _, _, grads = kept(model, image, target, weights, factors, steps, code, 64, c)
    norm2 = sum(float(np.sum(g[k].astype(np.float64) ** 2)) for g in grads for k in KEYS)
    eps = 1e-4 / np.sqrt(norm2)

    def loss(t):
        moved = [LevelWeights(**{k: getattr(w, k).astype(np.float64) + t * g[k] for k in KEYS})
                 for w, g in zip(weights, grads)]
        tape = oracle.train_forward(image, moved, channels=c, steps=steps, dtype=np.float64,
                                    ndim=ndim, n_in=n_in, factors=factors, seed=3, fire_rate=0.5)
        return oracle.readout_mse(tape.final, target)[0]
    slope = (loss(eps) - loss(-eps)) / (2 * eps)
    assert abs(slope / norm2 - 1) <= SLOPE[code]


def test_memory(gpu):
    """At 20 steps a level the kept step needs half the memory, with more less."""
    m = octnca.Model(ndim=2, n_in=3)
    f = [(1, 2, 2)] * 4
    part = []
    for n in (20, 64, 200):
        a = octnca.octree_nca_train_workspace_bytes(m, (1, 320, 320), f, [n] * 5)
        b = octnca.octree_nca_train_kept_workspace_bytes(m, (1, 320, 320), f, [n] * 5)
        part.append(b / a)
    assert part[0] < 0.55 and part[1] < 0.38 and part[2] < 0.31


def adamw_reference(w, g, state, t, lr, betas, eps, decay, max_norm, ema_decay):
    """One clipped update in float64, in place; returns the norm."""
    norm = np.sqrt(sum(float(np.sum(x ** 2)) for x in g))
    f = max_norm / norm if norm > max_norm else 1.0
    for i, x in enumerate(g):
        m, v, e = (state[k][i] for k in "mve")
        m += (1 - betas[0]) * (x * f - m)
        v += (1 - betas[1]) * ((x * f) ** 2 - v)
        w[i] -= lr * (m / (1 - betas[0] ** t) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
                      + decay * w[i])
        e += (1 - ema_decay) * (w[i] - e)
    return norm


@pytest.mark.parametrize("keep", [None, "i8", "f8"])
def test_trainer(gpu, keep):
    """Steps with updates: each follows the formulas from the gradients that the
    training step wrote, and the loss falls.  After one update a weight's error
    is the update's few fp32 roundings, at most 16 of 2^-24 of lr-sized and
    weight-sized terms; ten steps add up."""
    _, ndim, n_in, extent, factors, steps, c, h = CASES[0]
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h)
    model = octnca.Model(ndim=ndim, n_in=n_in)
    up = upload_weights(weights)
    lr = 2e-3
    tr = Trainer(model, extent, factors, steps, up, keep=keep, lr=lr, weight_decay=0.01,
                 max_norm=50.0)
    flat = lambda sets: [to_np(s[k]).astype(np.float64) for s in sets for k in KEYS]
    w = flat(up)
    state = {"m": [np.zeros_like(x) for x in w], "v": [np.zeros_like(x) for x in w],
             "e": [x.copy() for x in w]}
    losses = []
    for t in range(1, 11):
        loss, norm = tr.step(dev(image), dev(target), 0.5, 3)
        torch.cuda.synchronize()
        losses.append(float(loss))
        want = adamw_reference(w, flat(tr.grads), state, t, lr, (0.9, 0.99), 1e-8, 0.01, 50.0, 0.99)
        assert float(norm) == pytest.approx(want, rel=2.0 ** -22)
        for a, b, e, eb in zip(flat(up), w, flat(tr.ema), state["e"]):
            assert np.abs(a - b).max() <= t * 2.0 ** -20 * (np.abs(b).max() + lr)
            assert np.abs(e - eb).max() <= t * 2.0 ** -20 * (np.abs(b).max() + lr)
    assert int(tr.parameters.step) == 10
    assert losses[-1] < 0.9 * losses[0]


def test_trainer_leaves_out_a_step_that_overflowed(gpu):
    _, ndim, n_in, extent, factors, steps, c, h = CASES[0]
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h)
    up = upload_weights(weights)
    tr = Trainer(octnca.Model(ndim=ndim, n_in=n_in), extent, factors, steps, up, keep="i8")
    bad = target.copy()
    bad[0, 3, 3, 0] = np.inf
    before = [w["w1"].clone() for w in up]
    _, norm = tr.step(dev(image), dev(bad), 0.5, 3)
    assert not np.isfinite(float(norm)) and int(tr.parameters.step) == 0
    assert all(torch.equal(a, w["w1"]) for a, w in zip(before, up))
    _, norm = tr.step(dev(image), dev(target), 0.5, 3)
    assert np.isfinite(float(norm)) and int(tr.parameters.step) == 1


def test_trainer_on_another_stream(gpu):
    """A step on a stream of its own gives the same weights."""
    _, ndim, n_in, extent, factors, steps, c, h = CASES[5]
    image, target, weights = make(ndim, n_in, extent, factors, steps, c, h)
    model = octnca.Model(ndim=ndim, n_in=n_in)
    out = []
    for stream in (None, torch.cuda.Stream()):
        up = upload_weights(weights)
        tr = Trainer(model, extent, factors, steps, up, keep="i8", max_norm=1.0)
        x, y = dev(image), dev(target)
        torch.cuda.synchronize()
        for k in range(3):
            tr.step(x, y, 0.5, k, stream=stream)
        torch.cuda.synchronize()
        out.append([to_np(w[k]) for w in up for k in KEYS])
    assert all(np.array_equal(a, b) for a, b in zip(*out))


def test_refusals(gpu):
    m = octnca.Model(ndim=2, n_in=3)
    image, target, weights = make(2, 3, (1, 8, 8), (), (2,), 16, 64)
    up = upload_weights(weights)
    with pytest.raises(ValueError):
        Trainer(m, (1, 8, 8), (), (2,), up, keep="i4")
    for bad in (dict(steps=(-1,)), dict(factors=((1, 3, 2),), steps=(1, 1), weights=up * 2),
                dict(keep="i8", block=48), dict(model=octnca.Model(ndim=2, n_in=3, dtype="f16"))):
        args = dict(model=m, finest=(1, 8, 8), factors=(), steps=(2,), weights=up)
        with pytest.raises(octnca.OctreeNCAError):
            Trainer(**{**args, **bad})
    tr = Trainer(m, (1, 8, 8), (), (2,), up, keep="i8")
    tr.workspace = tr.workspace[:-256]
    with pytest.raises(octnca.OctreeNCAError) as e:
        tr.step(dev(image), dev(target), 0.5, 0)
    assert e.value.status == octnca.OCTNCA_ESPACE
    with pytest.raises(octnca.OctreeNCAError):
        tr.step(dev(image), dev(target)[..., :1], 0.5, 0)
