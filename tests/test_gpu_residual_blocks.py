"""The example that uses layer norm, feed-forward block, dropout and the SVGD step together: the scores it leaves in G are those that
autograd finds for the same network in plain torch, and training raises the likelihood."""
import os
import sys

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_scores_of_the_example():
    import residual_blocks
    n, width, rows, step = 3, 20, 37, 5
    net = residual_blocks.Ensemble(n, width, 48, 2, 0.25, seed=4)
    gen = torch.Generator().manual_seed(1)
    x, dy = torch.randn(rows, width, generator=gen).cuda(), torch.randn(n, rows, generator=gen).cuda()
    out, kept = net.forward(x.expand(n, -1, -1), step)
    dx = net.backward(dy, kept, step)

    leaves, s, start = [], x.double().cpu().expand(n, -1, -1).clone().requires_grad_(), 0
    first = s
    for b, (values, _) in enumerate(net.blocks):
        weight, bias, gate, up, down = p = [v.double().cpu().clone().requires_grad_() for v in values]
        leaves += p
        c = s - s.mean(-1, keepdim=True)
        h = c * (c.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * weight[:, None] + bias[:, None]
        z = (torch.nn.functional.silu(h @ gate.transpose(1, 2)) * (h @ up.transpose(1, 2))) @ down.transpose(1, 2)
        keep = ref.kept(n * rows * width, 0.25, 4, step * 2 + b).view(n, rows, width)
        s = s + torch.where(keep, z / 0.75, 0.0)
    readout = net.readout.double().cpu().clone().requires_grad_()
    want = (s @ readout.unsqueeze(2)).squeeze(2)
    (want * dy.double().cpu()).sum().backward()
    # two blocks of fp32 products over up to 96 values: some hundred roundings of 2^-24 of the largest terms
    assert (out.double().cpu() - want).abs().max() <= 2e-5 * want.abs().max()
    assert (dx.double().cpu() - first.grad).abs().max() <= 2e-5 * first.grad.abs().max()
    G = torch.cat([t.grad.reshape(n, -1) for t in (*leaves, readout)], 1)
    assert G.shape == net.G.shape
    assert (net.G.double().cpu() - G).abs().max() <= 2e-5 * G.abs().max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_training_raises_the_likelihood(dtype):
    import residual_blocks
    net, batch, y, history = residual_blocks.train(n=6, width=32, rows=128, steps=60, dtype=dtype, report=lambda line: None)
    assert torch.isfinite(history).all() and torch.isfinite(net.X).all()
    assert history[-5:].mean() > history[:5].mean()
    out, _ = net.forward(batch, train=False)
    assert out.shape == (6, 128) and out.std(0).mean() > 1e-3  # the particles have not collapsed onto one another
