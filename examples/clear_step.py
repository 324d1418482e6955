"""Training the paper's kind of network in the clear, on the card: an MLP whose hidden layers take 8-bit integers, as the encrypted
run's do, so that its results are what that run is compared with.

A step, next to the gadgets that do the same on ciphertexts:
  quantize_i8 + matmul_i8      the layers' products                    Matmul^RNS, Shift2MSBs
  linear_ce, linear_ce_grad    loss of the output layer, its gradient  IntCELossDeriv
  matmul_i8_grad               the layers' gradients                   Matmul^RNS, transposed
  orthogonalize                the update of the hidden weights        clipped weight update
and afterwards linear_i8 answers single inputs with the 8-bit weights.

  python examples/clear_step.py [--steps 60] [--batch 256]
Data is synthetic: classes are noisy copies of random patterns."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_17785_amd as slz  # noqa: E402


class Mlp:
    """Layers widths[0] -> ... -> widths[-1]; ReLU between them, the last one is the classifier's head."""

    def __init__(self, widths=(784, 128, 64, 10), dtype=torch.bfloat16, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = dtype
        self.weights = [torch.randn(n, k, device="cuda", generator=gen) * (2 / k) ** 0.5 for k, n in zip(widths, widths[1:])]
        self.momentum = [torch.zeros_like(w) for w in self.weights]

    def step(self, x, labels, rate=0.02, decay=0.9):
        """One training step on x [batch][inner]; the mean loss, on the card."""
        kept, h = [], x.to(self.dtype)
        for w in self.weights[:-1]:
            a, sa = slz.quantize_i8(h)
            b, sb = slz.quantize_i8(w)
            y = slz.matmul_i8(a, sa, b, sb, self.dtype)
            kept.append((a, sa, b, sb, y))
            h = y.relu()
        head = self.weights[-1].to(self.dtype)
        loss, lse = slz.linear_ce(h, head, labels)
        counts = (labels != -100).float()
        dh, dw = slz.linear_ce_grad(h, head, labels, lse, counts / counts.sum())
        grads = [dw]
        for i, (a, sa, b, sb, y) in reversed(list(enumerate(kept))):
            dh, dw = slz.matmul_i8_grad(dh * (y > 0), a, sa, b, sb, need_a=i > 0)
            grads.insert(0, dw)
        for i, (w, m, g) in enumerate(zip(self.weights, self.momentum, grads)):
            m.mul_(decay).add_(g.float())
            if i + 1 < len(self.weights):
                w.sub_(slz.orthogonalize(m.to(self.dtype)).float() * (rate * max(1.0, w.shape[0] / w.shape[1]) ** 0.5))
            else:
                w.sub_(m, alpha=10 * rate)
        return loss.sum() / counts.sum()

    def freeze(self):
        """8-bit weights of all layers with their scales: what is answered with."""
        return [slz.quantize_i8(w) for w in self.weights]


def answer(frozen, x, dtype=torch.bfloat16):
    """Logits [rows][classes] by 8-bit products alone."""
    h = x.to(dtype)
    for i, (q, scale) in enumerate(frozen):
        h = slz.linear_i8(h, q, scale)
        if i + 1 < len(frozen):
            h = h.relu()
    return h


def synthetic(count, inner=784, classes=10, seed=7):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    patterns = torch.randn(classes, inner, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    labels = torch.randint(0, classes, (count,), device="cuda", generator=gen)
    return patterns[labels] * 0.3 + torch.randn(count, inner, device="cuda", generator=gen), labels


def train(steps=60, batch=256):
    net, losses = Mlp(), []
    for i in range(steps):
        x, labels = synthetic(batch, seed=100 + i)
        losses.append(net.step(x, labels))
    frozen = net.freeze()
    x, labels = synthetic(2048, seed=5)
    right = (answer(frozen, x).argmax(1) == labels).float().mean()
    one = answer(frozen, x[:1])
    return [float(v) for v in losses], float(right), one, answer(frozen, x)[:1]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=256)
    a = ap.parse_args()
    losses, right, _, _ = train(a.steps, a.batch)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.4f" % (i, losses[i]))
    print("8-bit network: %.1f %% of 2048 new inputs right (one in ten by chance)" % (100 * right))


if __name__ == "__main__":
    main()
