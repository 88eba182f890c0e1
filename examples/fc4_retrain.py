"""Compress two fully-connected layers to 4 bits, retrain what 4 bits leave open, and serve single tokens.

The weights' 16 levels come from the framework's k-means over scalars (kq_quantize_scalars) on the weights divided
by their group's largest; the group scales are then retrained against the uncompressed layers: forward from the
codes with the inputs kept as 8-bit checkpoints, backward through the codes to the hidden activation and from the
checkpoints to the scales and biases.  Synthetic weights and activations.

    python examples/fc4_retrain.py [--steps 30] [--in 4096 --hidden 4096 --out 1000] [--batch 256]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2003_05148_amd as kq  # noqa: E402


def group_levels(W, group):
    """16 bf16 levels: k-means over the weights divided by the largest magnitude of their group."""
    n, k = W.shape
    g = torch.nn.functional.pad(W, (0, -k % group)).view(n, -1, group)
    unit = (g / g.abs().amax(2, keepdim=True).clamp(min=1e-30)).view(n, -1)[:, :k].contiguous()
    _, levels, _, _ = kq.kq_quantize_scalars(unit, bits=4, want_v_hat=False)
    return levels.sort().values.to(torch.bfloat16)


def retrain(n_in=4096, n_hidden=4096, n_out=1000, batch=256, steps=30, group=128, gamma=None, seed=0):
    """Returns (losses, the two layers): the mean squared error of the 4-bit layers' output against the
    uncompressed layers' at every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    W1, b1 = randn(n_hidden, n_in) / math.sqrt(n_in), 0.1 * randn(n_hidden)
    W2, b2 = randn(n_out, n_hidden) / math.sqrt(n_hidden), 0.1 * randn(n_out)
    fc1 = kq.GroupLinear(W1, group, group_levels(W1, group), b1)
    fc2 = kq.GroupLinear(W2, group, group_levels(W2, group), b2)
    gamma = gamma if gamma is not None else 0.02 * group / 128
    losses = []
    for _ in range(steps):
        X = randn(batch, n_in).relu_().to(torch.bfloat16)
        want = torch.relu(X.float() @ W1.t() + b1) @ W2.t() + b2
        H, ck1 = fc1.forward(X)
        A = torch.relu(H)
        Y, ck2 = fc2.forward(A)
        diff = Y.float() - want
        losses.append(float((diff * diff).mean()))
        dY = (diff * (2.0 / batch)).to(torch.bfloat16)      # of the sum over outputs of the mean over the batch
        dA, ds2, db2 = fc2.backward(dY, ck2)
        _, ds1, db1 = fc1.backward(torch.where(A > 0, dA, 0), ck1, input_grad=False)
        # a scale's curvature is its group's mean of (level * input)^2: steps in units of it
        fc2.step(ds2 / group, db2, gamma)
        fc1.step(ds1 / group, db1, gamma)
    return losses, (fc1, fc2)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--in", dest="n_in", type=int, default=4096)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--out", type=int, default=1000)
    p.add_argument("--batch", type=int, default=256)
    a = p.parse_args()
    losses, (fc1, fc2) = retrain(a.n_in, a.hidden, a.out, a.batch, a.steps)
    print(f"mean squared error: {losses[0]:.3e} after quantization, {losses[-1]:.3e} after {a.steps} steps")
    token = torch.randn(1, a.n_in, device="cuda").relu_().to(torch.bfloat16)
    for _ in range(3):
        fc2(torch.relu(fc1(token)))
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    for _ in range(100):
        y = fc2(torch.relu(fc1(token)))
    t1.record()
    torch.cuda.synchronize()
    print(f"one token through both layers: {t0.elapsed_time(t1) * 10:.1f} us, output {tuple(y.shape)}")


if __name__ == "__main__":
    main()
