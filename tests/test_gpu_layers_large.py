"""The particles' layers at sizes beyond those of test_gpu_layers.py: every tile and every way of splitting sums that the feed-forward
block's sizes lead to, and offsets that pass 32 bits."""
import pytest
import torch

import layer_reference as ref
from test_gpu_layers import IDS, TYPES, acts, gen, layers, params, run_ffn  # noqa: F401

pytestmark = pytest.mark.gpu

# The smallest of some ten thousand random shapes that take, in this order: large and small tiles of h down^T, whole and with its columns in
# parts; large and small ones of g and u; of the gradients, with their columns whole, in parts for dx, for the parameters and for both; of dh.
TILED = [(40, 1_028, 133, 83), (24, 77, 665, 1_602), (5, 3_501, 66, 43), (24, 70, 208, 513), (40, 741, 32, 68), (13, 3_361, 34, 35), (24, 453, 203, 165),
         (5, 70, 502, 595), (8, 1_910, 130, 103), (1, 3_413, 403, 1_039), (64, 267, 67, 135), (40, 73, 107, 309), (3, 4_629, 72, 44), (2, 2_865, 197, 401),
         (8, 3_862, 44, 131), (8, 5_985, 32, 66)]
# The same for the gradients with later rates: large tiles whole and with the parameters' rows in parts, small ones with these in parts, and with both,
# the smallest with both.
TILED += [(64, 227, 199, 122), (8, 3_543, 133, 105), (5, 5_030, 74, 46), (3, 1_769, 198, 474), (1, 284, 46, 135)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,hidden", TILED)
def test_ffn_every_tile(layers, n, rows, width, hidden, dtype):  # noqa: F811
    g = gen(n, rows, width, hidden)
    x, dy = acts(g, n, rows, width, dtype, "gap"), acts(g, n, rows, width, dtype)
    p, grads, G, D = params(g, n, 3, (hidden, width), (hidden, width), (width, hidden), spread=width ** -0.5)
    got, want = run_ffn(layers, x, dy, p, grads, "silu"), ref.gated_ffn(x, *p, "silu", dy)
    for name in want:
        ref.check(got[name], want[name], f"{name} of {n}x{rows}x{width}x{hidden}")
    assert (G[:, :3] == -7.0).all() and (G[:, D - 3:] == -7.0).all()
    first = [t.clone() for t in grads]
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    assert torch.equal(y, got["y"])
    layers.gated_ffn_backward(dy, x, *p, saved, *grads, accumulate=True, want_dx=False)
    assert all(torch.equal(t, 2 * f) for t, f in zip(grads, first))


def positive(*shape, dtype=torch.float32, seed=0):
    return (torch.rand(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") + 0.5).to(dtype)


def test_ffn_far_rows(layers):  # noqa: F811
    """g, u and h of more than 2^31 values.  Everything is positive, so sums over the rows are what their terms' absolute values add up to, and
    the 6 % of the rows beyond 2^31 values show in them: sums of 32 rows at a time are off by at most rows / 32 + 64 roundings."""
    rows, width, hidden = (1 << 22) + 3, 8, 520
    x, dy = positive(1, rows, width, dtype=torch.bfloat16, seed=1), positive(1, rows, width, dtype=torch.bfloat16, seed=2)
    gate, up, down = (positive(1, *s, seed=3 + k) * 0.1 for k, s in enumerate(((hidden, width), (hidden, width), (width, hidden))))
    y, saved = layers.gated_ffn_forward(x, gate, up, down, save=True)
    assert saved.numel() // 3 > 1 << 31
    grads = [torch.full_like(t, float("nan")) for t in (gate, up, down)]
    dx = layers.gated_ffn_backward(dy, x, gate, up, down, saved, *grads)
    del saved
    for part in (slice(0, 40), slice(rows - 40, rows)):
        want = ref.gated_ffn(x[:, part], gate, up, down, "silu", dy[:, part])
        ref.check(y[:, part], want["y"], "y")
        ref.check(dx[:, part], want["dx"], "dx")
    sums = [torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((hidden, width), (hidden, width), (width, hidden))]
    for start in range(0, rows, 1 << 18):
        a, d = x[0, start:start + (1 << 18)].double(), dy[0, start:start + (1 << 18)].double()
        g, u = a @ gate[0].double().t(), a @ up[0].double().t()
        act, slope, _, _ = ref.activation(g, "silu")
        dh = d @ down[0].double()
        sums[0] += (dh * u * slope).t() @ a
        sums[1] += (dh * act).t() @ a
        sums[2] += d.t() @ (act * u)
    for got, want in zip(grads, sums):
        assert ((got[0].double() - want).abs() <= (rows / 32 + 64) * ref.U * want).all()


def test_norm_far_rows(layers):  # noqa: F811
    """Activations of more than 2^31 values; dy = x, so that dweight is a sum of positive terms on the whole, and dbias of positive ones."""
    rows, width = (1 << 20) + 5, 2_056
    assert rows * width > 1 << 31
    x = positive(1, rows, width, dtype=torch.bfloat16, seed=1)
    w, b = positive(1, width, seed=2), positive(1, width, seed=3)
    y, mean, rstd = layers.layer_norm_forward(x, w, b)
    dw, db = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    dx = layers.layer_norm_backward(x, x, w, mean, rstd, dw, db)
    for part in (slice(0, 40), slice(rows - 40, rows)):
        want = ref.layer_norm(x[:, part], w, b, 1e-5, x[:, part])
        ref.check(y[:, part], want["y"], "y")
        ref.check(dx[:, part], want["dx"], "dx")
    sums, size = torch.zeros(2, width, dtype=torch.float64, device="cuda"), torch.zeros(width, dtype=torch.float64, device="cuda")
    for start in range(0, rows, 1 << 16):
        v = x[0, start:start + (1 << 16)].double()
        c = v - v.mean(-1, keepdim=True)
        t = v * c * ((c * c).mean(-1, keepdim=True) + 1e-5).rsqrt()
        sums[0] += t.sum(0)
        sums[1] += v.sum(0)
        size += t.abs().sum(0)
    # at least 256 workgroups add up at most rows / 256 + 1 values one by one; a value of xhat is off by some width / 64 + 20 roundings
    bound = (rows / 256 + 64) * ref.U
    assert ((dw[0].double() - sums[0]).abs() <= (bound + 64 * ref.U) * size).all()
    assert ((db[0].double() - sums[1]).abs() <= bound * sums[1]).all()


def test_parameters_far_out_in_a_row(layers):  # noqa: F811
    """The layers' parameters and gradients behind 2^31 others of each particle."""
    n, rows, width, hidden, at = 2, 5, 24, 40, (1 << 31) + 7
    X, G = torch.empty(n, at + 4_000, device="cuda"), torch.empty(n, at + 4_000, device="cuda")
    g = gen(21)
    views = []
    for size in (width, width, hidden * width, hidden * width, width * hidden):
        X[:, at:at + size] = torch.randn(n, size, generator=g).cuda() * 0.3
        views.append((X[:, at:at + size], G[:, at:at + size]))
        at += size
    (w, dw), (b, db) = views[:2]
    p, grads = zip(*((v.view(n, *s), d.view(n, *s)) for (v, d), s in zip(views[2:], ((hidden, width), (hidden, width), (width, hidden)))))
    for count in (rows, 70):
        x, dy = acts(g, n, count, width, torch.float32), acts(g, n, count, width, torch.float32)
        got, want = run_ffn(layers, x, dy, p, grads, "gelu"), ref.gated_ffn(x, *p, "gelu", dy)
        for name in want:
            ref.check(got[name], want[name], name)
        y, mean, rstd = layers.layer_norm_forward(x, w, b)
        dx = layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db)
        want = ref.layer_norm(x, w, b, 1e-5, dy)
        for name, t in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
            ref.check(t, want[name], name)


def test_no_grad_keeps_nothing(layers):  # noqa: F811
    """Without gradients the block as an autograd function takes the memory of the plain call: g and u are not kept."""
    x, w = torch.randn(2, 500, 64, device="cuda"), torch.randn(2, 64, device="cuda", requires_grad=True)
    gate, down = torch.randn(2, 256, 64, device="cuda", requires_grad=True), torch.randn(2, 64, 256, device="cuda", requires_grad=True)

    def peak(f):
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = f()
        return out, torch.cuda.max_memory_allocated() - before

    with torch.no_grad():
        a, plain = peak(lambda: layers.gated_ffn_forward(x, gate, gate, down)[0])
        b, function = peak(lambda: layers.gated_ffn(x, gate, gate, down))
        assert torch.equal(a, b) and not b.requires_grad and function <= plain
        assert torch.equal(layers.layer_norm(x, w), layers.layer_norm_forward(x, w)[0])
        assert torch.equal(layers.dropout(x, 0.3, 1), layers.dropout_forward(x, 0.3, 1))
    c = layers.gated_ffn(x, gate, gate, down)
    assert torch.equal(a, c) and c.requires_grad
