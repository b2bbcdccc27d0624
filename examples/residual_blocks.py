#!/usr/bin/env python3
"""An ensemble of residual feed-forward networks trained with SVGD, start to end on the n x D matrices.

Every particle is a network of `--blocks` residual blocks s <- s + dropout(ffn(layer_norm(s))) and a linear read-out,
trained on one shared regression batch (Gaussian likelihood, Gaussian prior).  All parameters of particle i lie in row i of X;
the backward pass leaves its score in row i of G, where svgd.Svgd.step reads it: nothing is packed or copied in between,
and each block is one call per layer for all particles.

    python examples/residual_blocks.py [--particles 8] [--width 64] [--blocks 2] [--rows 256] [--steps 100]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_06528_amd import layers, svgd  # noqa: E402


class Ensemble:
    """n residual networks as views into the rows of X, with their scores as views into the rows of G."""

    def __init__(self, n, width, hidden, blocks, p, seed, dtype=torch.float32):
        self.n, self.width, self.hidden, self.p, self.seed, self.dtype = n, width, hidden, p, seed, dtype
        shapes = []
        for _ in range(blocks):
            shapes += [(width,), (width,), (hidden, width), (hidden, width), (width, hidden)]
        shapes.append((width,))  # the read-out
        D = sum(math.prod(s) for s in shapes)
        self.X, self.G = svgd.padded_rows(n, D, fill=0.0), svgd.padded_rows(n, D, fill=0.0)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        values, grads, at = [], [], 0
        for s in shapes:
            size = math.prod(s)
            value = self.X[:, at:at + size].view(n, *s)
            if len(s) > 1:
                value.copy_(torch.randn(n, *s, generator=gen, device="cuda") * s[-1] ** -0.5)
            values.append(value)
            grads.append(self.G[:, at:at + size].view(n, *s))
            at += size
        self.blocks = [(values[k:k + 5], grads[k:k + 5]) for k in range(0, 5 * blocks, 5)]
        for (weight, *_), _ in self.blocks:
            weight.fill_(1.0)
        self.readout, self.readout_grad = values[-1], grads[-1]
        self.readout.copy_(torch.randn(n, width, generator=gen, device="cuda") * width ** -0.5)

    def forward(self, x, step=0, train=True):
        """The predictions (n, rows) for inputs (n, rows, width), and what the backward pass needs.  In prediction dropout is off
        (p = 0 would do as well, but a whole pass over the stream would go into it)."""
        kept, s = [], x
        for b, ((weight, bias, gate, up, down), _) in enumerate(self.blocks):
            h, mean, rstd = layers.layer_norm_forward(s, weight, bias)
            z, saved = layers.gated_ffn_forward(h, gate, up, down, save=train)
            kept.append((s, h, mean, rstd, saved))
            s = layers.dropout_forward(z, self.p, self.seed, step * len(self.blocks) + b, residual=s) if train else s + z
        kept.append(s)
        return (s.float() @ self.readout.unsqueeze(2)).squeeze(2), kept

    def backward(self, dy, kept, step=0):
        """Scores into G from the gradient dy (n, rows) of the log likelihood by the predictions; the gradient by the inputs."""
        s = kept[-1]
        self.readout_grad.copy_((dy.unsqueeze(1) @ s.float()).squeeze(1))
        ds = (dy.unsqueeze(2) * self.readout.unsqueeze(1)).to(self.dtype)
        for b in reversed(range(len(self.blocks))):
            (weight, _, gate, up, down), (dweight, dbias, dgate, dup, ddown) = self.blocks[b]
            s, h, mean, rstd, saved = kept[b]
            dz = layers.dropout_backward(ds, self.p, self.seed, step * len(self.blocks) + b)
            dh = layers.gated_ffn_backward(dz, h, gate, up, down, saved, dgate, dup, ddown)
            ds = ds + layers.layer_norm_backward(dh, s, weight, mean, rstd, dweight, dbias)
        return ds


def train(n=8, width=64, blocks=2, rows=256, steps=100, lr=2e-3, p=0.1, noise=0.1, prior=1.0, seed=0, dtype=torch.float32, report=print):
    """The ensemble and its mean log likelihood per step."""
    net = Ensemble(n, width, (8 * width // 3 + 31) // 32 * 32, blocks, p, seed, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(rows, width, generator=gen, device="cuda")
    y = torch.sin(2.0 * x[:, 0]) * x[:, 1]
    batch = x.to(dtype).expand(n, -1, -1)  # every particle sees the same rows
    history = []
    with svgd.Svgd(n, net.X.shape[1]) as engine:
        for step in range(steps):
            out, kept = net.forward(batch, step)
            residual = y - out
            net.backward(residual / (noise * noise * rows), kept, step)  # of the mean log likelihood
            net.G.sub_(net.X, alpha=1.0 / (prior * prior * rows))
            engine.step(net.X, net.G, lr)
            history.append(-0.5 * (residual * residual).mean() / (noise * noise))
            if step % max(1, steps // 10) == 0:
                report(f"step {step:4d}  log likelihood per row {history[-1].item():9.3f}")
    return net, batch, y, torch.stack(history)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("particles", 8), ("width", 64), ("blocks", 2), ("rows", 256), ("steps", 100)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    net, batch, y, history = train(a.particles, a.width, a.blocks, a.rows, a.steps)
    out, _ = net.forward(batch, train=False)
    print(f"posterior mean's squared error {((out.mean(0) - y) ** 2).mean().item():.4f}, spread of the particles {out.std(0).mean().item():.4f}")


if __name__ == "__main__":
    main()
