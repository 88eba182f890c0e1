"""Put a classifier's two fully-connected layers into 8-bit floats, retrain them against the uncompressed classifier, and serve
single tokens.

The weights become e4m3 values with a power of two for each 128 x 128 block (BlockLinear); of the uncompressed
classifier only every row's largest logits are kept, and the 8-bit layers are distilled from those and the labels:
forward from 8-bit values that the weights' gradients are taken from again, the loss and the gradient of the logits in one
pass, backward through the 8-bit weights.  Synthetic weights, activations and labels.

    python examples/fc8_distill.py [--steps 30] [--in 4096 --hidden 4096 --classes 1000] [--batch 256]
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


def gradients(fc1, fc2, X, top_values, top_idx, labels, temperature=2.0, alpha=0.3):
    """(loss of every row, gradients of the mean loss (dW1, db1, dW2, db2)) of two layers with a ReLU between them."""
    H, kept1 = fc1.forward(X)
    Z, kept2 = fc2.forward(torch.relu(H))
    loss, dZ = kq.kq_distill(Z, top_values, top_idx, temperature, labels, alpha, scale=1.0 / X.shape[0])
    dA, dW2, db2 = fc2.backward(dZ, kept2)
    _, dW1, db1 = fc1.backward(torch.where(H > 0, dA, 0), kept1, input_grad=False)
    return loss, (dW1, db1, dW2, db2)


def retrain(n_in=4096, n_hidden=4096, classes=1000, batch=256, steps=30, top=10, gamma=0.005, seed=0):
    """Returns (mean loss of every step, the two layers)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    W1, b1 = randn(n_hidden, n_in) / math.sqrt(n_in), 0.1 * randn(n_hidden)
    W2, b2 = 4 * randn(classes, n_hidden) / math.sqrt(n_hidden), 0.1 * randn(classes)
    fc1, fc2 = kq.BlockLinear(W1, b1, master=True), kq.BlockLinear(W2, b2, master=True)
    losses = []
    for _ in range(steps):
        X = randn(batch, n_in).relu_().to(torch.bfloat16)
        teacher = torch.relu(X.float() @ W1.t() + b1) @ W2.t() + b2
        top_values, top_idx = teacher.topk(top, dim=1)
        loss, (dW1, db1, dW2, db2) = gradients(fc1, fc2, X, top_values, top_idx, top_idx[:, 0].contiguous())
        losses.append(float(loss.mean()))
        fc2.step(dW2, db2, gamma)
        fc1.step(dW1, db1, gamma)
    return losses, (fc1, fc2)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--in", dest="n_in", type=int, default=4096)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--classes", type=int, default=1000)
    p.add_argument("--batch", type=int, default=256)
    a = p.parse_args()
    losses, (fc1, fc2) = retrain(a.n_in, a.hidden, a.classes, a.batch, a.steps)
    print(f"mean loss: {losses[0]:.4f} after quantization, {losses[-1]:.4f} after {a.steps} steps")
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
