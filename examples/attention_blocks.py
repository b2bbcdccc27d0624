#!/usr/bin/env python3
"""An ensemble of small causal transformers trained with SVGD, start to end on the n x D matrices.

Every particle is a network of `--blocks` blocks

    s <- s + linear(attention(qk_norm_rotary(linear(layer_norm(s)))))
    s <- s + ffn(layer_norm(s))

and a linear read-out of every token, trained on one shared batch of sequences (Gaussian likelihood, Gaussian prior): the running mean of a signal that each token shows with noise.
All parameters of particle i lie in row i of X, autograd leaves its score in row i of G, where svgd.Svgd.step reads it.  Afterwards the sequences are continued token by token over caches of keys
and values, which gives what the whole sequence gives.

    python examples/attention_blocks.py [--particles 8] [--width 64] [--blocks 2] [--batch 8] [--tokens 48] [--steps 60]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_06528_amd import attention as att  # noqa: E402
from paper_2306_06528_amd import layers, svgd  # noqa: E402


class Ensemble:
    """n transformers as views into the rows of X: leaves of autograd whose gradients are views into the rows of G."""

    def __init__(self, n, width, blocks, seed, heads=4, kv_heads=2, dtype=torch.float32):
        self.n, self.width, self.heads, self.kv, self.dim, self.dtype = n, width, heads, kv_heads, width // heads, dtype
        hidden = (8 * width // 3 + 31) // 32 * 32
        qkv = (heads + 2 * kv_heads) * self.dim
        block = {"norm1": (width,), "bias1": (width,), "qkv": (qkv, width), "qkv_bias": (qkv,), "q_norm": (self.dim,), "k_norm": (self.dim,), "slopes": (heads,), "out": (width, width),
                 "norm2": (width,), "bias2": (width,), "gate": (hidden, width), "up": (hidden, width), "down": (width, hidden)}
        shapes = [(b, k, s) for b in range(blocks) for k, s in block.items()] + [(None, "readout", (1, width))]
        D = sum(math.prod(s) for _, _, s in shapes)
        self.X, self.G = svgd.padded_rows(n, D, fill=0.0), svgd.padded_rows(n, D, fill=0.0)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.blocks, self.leaves, at = [{} for _ in range(blocks)], [], 0
        for b, name, shape in shapes:
            size = math.prod(shape)
            value = self.X[:, at:at + size].view(n, *shape)
            if "norm" in name:
                value.fill_(1.0)
            elif len(shape) > 1:
                value.copy_(torch.randn(n, *shape, generator=gen, device="cuda") * shape[-1] ** -0.5)
            elif name == "slopes":
                value.copy_(torch.exp2(-8.0 * torch.arange(1, heads + 1, device="cuda") / heads).expand(n, -1))
            leaf = value.detach().requires_grad_()
            leaf.grad = self.G[:, at:at + size].view(n, *shape)
            self.leaves.append(leaf)
            if b is None:
                self.readout = leaf
            else:
                self.blocks[b][name] = leaf
            at += size
        self.frequencies = torch.tensor([10_000.0 ** (-2 * j / self.dim) for j in range(self.dim // 2)], dtype=torch.float64, device="cuda")

    def block(self, p, s, batch, positions, cache=None):
        """s is (n, batch * tokens, width).  With a cache, (keys, values, how many there are of each sequence), these tokens' are added to it."""
        n, d, tokens = self.n, self.dim, s.shape[1] // batch
        h = layers.layer_norm(s, p["norm1"], p["bias1"])
        qkv = att.linear(h, p["qkv"], p["qkv_bias"]).view(n, batch, tokens, self.heads + 2 * self.kv, d)
        q, k, v = qkv[..., :self.heads, :], qkv[..., self.heads:self.heads + self.kv, :], qkv[..., self.heads + self.kv:, :]
        q, k = att.qk_norm_rotary(q, k, p["q_norm"], p["k_norm"], self.frequencies, positions)
        if cache is None:
            o = att.attention(q, k, v, causal=True, slopes=p["slopes"])
        else:
            keys, values, filled = cache
            first = int(positions[0])
            keys[:, :, first:first + tokens], values[:, :, first:first + tokens] = k, v
            filled += tokens
            o = att.attention(q, keys, values, causal=True, slopes=p["slopes"], lengths=filled, starts=filled - tokens)
        s = att.linear(o.view(n, batch * tokens, self.heads * d), p["out"], residual=s)
        return s + layers.gated_ffn(layers.layer_norm(s, p["norm2"], p["bias2"]), p["gate"], p["up"], p["down"])

    def forward(self, x, start=0, caches=None):
        """Predictions (n, batch, tokens) for x (batch, tokens, width); with caches, of tokens that follow `start` others."""
        batch, tokens = x.shape[:2]
        positions = torch.arange(start, start + tokens, device="cuda")
        s = x.to(self.dtype).reshape(1, batch * tokens, self.width).expand(self.n, -1, -1)
        for b, p in enumerate(self.blocks):
            s = self.block(p, s, batch, positions, caches and caches[b])
        return att.linear(s, self.readout).view(self.n, batch, tokens)

    def caches(self, batch, tokens):
        new = lambda: torch.empty(self.n, batch, tokens, self.kv, self.dim, dtype=self.dtype, device="cuda")  # noqa: E731
        return [(new(), new(), torch.zeros(batch, dtype=torch.int32, device="cuda")) for _ in self.blocks]

    def continued(self, x, prompt):
        """The same predictions, a prompt first and then token by token."""
        with torch.no_grad():
            caches = self.caches(*x.shape[:2])
            out = [self.forward(x[:, :prompt], 0, caches)]
            out += [self.forward(x[:, t:t + 1], t, caches) for t in range(prompt, x.shape[1])]
        return torch.cat(out, 2)


def train(n=8, width=64, blocks=2, batch=8, tokens=48, steps=60, lr=2e-3, noise=0.1, prior=1.0, seed=0, dtype=torch.float32, report=print):
    """The ensemble and its mean log likelihood per step."""
    net = Ensemble(n, width, blocks, seed, dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(batch, tokens, width, generator=gen, device="cuda")
    y = x[..., 0].cumsum(1) / torch.arange(1, tokens + 1, device="cuda").sqrt()
    history = []
    with svgd.Svgd(n, net.X.shape[1]) as engine:
        for step in range(steps):
            net.G.zero_()
            residual = y - net.forward(x).float()
            value = -0.5 * (residual * residual).mean((1, 2)) / (noise * noise)
            value.sum().backward()
            net.G.sub_(net.X, alpha=1.0 / (prior * prior * batch * tokens))
            engine.step(net.X, net.G, lr)
            history.append(value.detach().mean())
            if step % max(1, steps // 10) == 0:
                report(f"step {step:4d}  log likelihood per token {history[-1].item():9.3f}")
    return net, x, y, torch.stack(history)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("particles", 8), ("width", 64), ("blocks", 2), ("batch", 8), ("tokens", 48), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    net, x, y, history = train(a.particles, a.width, a.blocks, a.batch, a.tokens, a.steps)
    with torch.no_grad():
        out = net.forward(x)
    print(f"posterior mean's squared error {((out.mean(0) - y) ** 2).mean().item():.4f}, spread of the particles {out.std(0).mean().item():.4f}")
    print(f"token by token: largest difference {(net.continued(x, a.tokens // 2) - out).abs().max().item():.2e}")


if __name__ == "__main__":
    main()
