"""Training on synthetic pathology patches: gradients of a training step, the
clipped AdamW update and a running average of the weights, with every state kept
in fp32 or in 8 bits.

    python examples/train_patches.py                    # 320 x 320, states in fp32
    python examples/train_patches.py --keep i8          # the same, states in 8 bits
    python examples/train_patches.py --size 1280 --nca-steps 64 --keep i8
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_06993_amd as octnca                                     # noqa: E402
from paper_2508_06993_amd.runtime import Trainer, upload_weights          # noqa: E402
from synthetic import TRAIN_WORKLOADS, make_image, make_target, make_weights, scaled   # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--size", type=int, default=320, help="rows and columns of a patch")
    ap.add_argument("--nca-steps", type=int, default=20, help="NCA steps per level")
    ap.add_argument("--patches", type=int, default=4, help="patches to go through in turn")
    ap.add_argument("--steps", type=int, default=40, help="training steps")
    ap.add_argument("--keep", default="f32", choices=["f32", "i8", "f8"],
                    help="how the states for the backward are kept")
    ap.add_argument("--lr", type=float, default=1.6e-3)
    ap.add_argument("--max-norm", type=float, default=1.0)
    args = ap.parse_args(argv)

    base = TRAIN_WORKLOADS["pathology_train320"]
    wl = scaled(base, (1, args.size, args.size), steps=(args.nca_steps,) * base.levels,
                factors=base.factors)
    images = [make_image(wl, k) for k in range(args.patches)]
    data = [(torch.from_numpy(x).cuda(), torch.from_numpy(make_target(wl, x)).cuda())
            for x in images]
    # random weights of a tenth of the workloads' magnitude: states stay near the image's
    weights = upload_weights([{k: 0.1 * getattr(w, k) for k in ("conv_w", "conv_b", "w1", "b1", "w2")}
                              for w in make_weights(wl)])
    trainer = Trainer(octnca.Model(ndim=wl.ndim, n_in=wl.n_in), wl.extent, wl.factors, wl.steps,
                      weights, keep=None if args.keep == "f32" else args.keep, lr=args.lr,
                      max_norm=args.max_norm)
    cells = args.size * args.size
    start = None
    for k in range(args.steps):
        loss, norm = trainer.step(*data[k % len(data)], wl.fire_rate, seed=k)
        if k % 10 == 0 or k == args.steps - 1:
            print(f"step {k}: loss per cell {float(loss) / cells:.5f}, gradient norm "
                  f"{float(norm):.3g}", flush=True)
        if k == 0:       # the first step has loaded the kernels
            start = time.perf_counter()
    torch.cuda.synchronize()
    ms = (time.perf_counter() - start) / max(1, args.steps - 1) * 1e3
    print(f"{ms:.3f} ms a step, workspace {trainer.workspace.numel() / 1e6:.1f} MB", flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
