"""What the layers' header says about precision, at inputs that show it."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_layers import IDS, TYPES, gen, layers  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows", [5, 32, 70, 1_000])
def test_ffn_products_are_those_of_fp32_whatever_the_type(layers, rows, dtype):  # noqa: F811
    """y and dx of two terms each that cancel but for 2^-12 of them.  x and dy are unit rows, so g, u and dh are the parameters' values
    themselves: h, dg and du are off by at most ten roundings of fp32, and two products in fp32, each as six of parts that are added up one by one, by
    sixteen more; then the result is rounded to its type.  (Operands of 16 bits would be off by 2^-17 each.)"""
    g = gen(31)
    n, width, hidden = 3, 200, 70
    gate, up, down = torch.zeros(n, hidden, width), torch.zeros(n, hidden, width), torch.zeros(n, width, hidden)
    gate[:, :, 0] = torch.rand(n, hidden, generator=g) + 0.5
    up[:, :, 0] = torch.rand(n, hidden, generator=g) + 0.5
    gv, uv = gate[:, :2, 0].double(), up[:, :2, 0].double()
    a, slope, _, _ = ref.activation(gv, "silu")
    h = a * uv
    near = 1.0 + 2.0 ** -12
    down[:, :, 0] = torch.rand(n, width, generator=g) + 0.5
    down[:, :, 1] = (-near * (h[:, :1] / h[:, 1:]) * down[:, :, 0].double()).float()
    dg, du = (down[:, 0, :2].double() * t for t in (uv * slope, a))
    for d, w, cols in ((dg, gate, slice(1, 100)), (du, up, slice(100, 200))):  # (where x is 0)
        w[:, 0, cols] = torch.rand(n, cols.stop - cols.start, generator=g) + 0.5
        w[:, 1, cols] = (-near * (d[:, :1] / d[:, 1:]) * w[:, 0, cols].double()).float()
    x = torch.zeros(n, rows, width, dtype=dtype)
    x[:, :, 0] = 1.0
    want = {"y": down[:, :, :2].double() @ h.unsqueeze(2), "dx": gate[:, :2].double().transpose(1, 2) @ dg.unsqueeze(2) + up[:, :2].double().transpose(1, 2) @ du.unsqueeze(2)}
    size = {"y": down[:, :, :2].double().abs() @ h.abs().unsqueeze(2),
            "dx": gate[:, :2].double().abs().transpose(1, 2) @ dg.abs().unsqueeze(2) + up[:, :2].double().abs().transpose(1, 2) @ du.abs().unsqueeze(2)}
    x, gate, up, down = (t.cuda() for t in (x, gate, up, down))
    y, saved = layers.gated_ffn_forward(x, gate, up, down, save=True)
    got = {"y": y, "dx": layers.gated_ffn_backward(x, x, gate, up, down, saved)}
    for name in got:
        v = want[name].transpose(1, 2)
        assert v[:, :, 1:].abs().max() < 1e-3
        ref.check(got[name], (v.expand(n, rows, width), (ref.rounding(dtype) * v.abs() + 26 * ref.U * size[name].transpose(1, 2)).expand(n, rows, width)), name)


@pytest.mark.parametrize("width", [7, 48, 200, 384, 1_001, 2_000, 5_003, 16_001])
def test_norm_of_rows_very_far_from_zero(layers, width):  # noqa: F811
    """Rows at 1e5: one of equal values, whose result is the bias, and one with a spread of 0.1, twelve steps of fp32.  The first mean is off by at most E + 16 roundings
    of 1e5 (E <= 16 values to a thread, 10 halvings), at most 0.2; what is taken off a second time is the mean of such distances, exact differences, to as many roundings of it, 4e-7, and rstd
    is at most 317 for the first row."""
    g = gen(32, width)
    x = torch.full((1, 2, width), 1e5 + 0.3)
    x[0, 1] += torch.randn(width, generator=g) * 0.1
    w, b = torch.rand(1, width, generator=g) + 0.5, torch.rand(1, width, generator=g)
    y, mean, rstd = (t.double().cpu() for t in layers.layer_norm_forward(x.cuda(), w.cuda(), b.cuda(), 1e-5))
    assert ((y[0, 0] - b[0].double()).abs() <= 4e-7 * 317 * w[0].double() + 2 * ref.U * b[0].double()).all()
    exact = x[0].double()
    m = exact.mean(-1)
    assert ((mean[0] - m).abs() <= 2 * ref.U * m).all()
    c = exact[1] - m[1]
    r = (c.square().mean() + 1e-5).rsqrt()
    want = c * r * w[0].double() + b[0].double()
    # (the second row's variance: some 1e-2, off by the square of 4e-7 and E + 20 roundings of it and of the square that is taken off, at most 0.04)
    off = 4e-7 * r * w[0].double() + 36 * ref.U * 5 * (want.abs() + b[0].double())
    assert ((y[0, 1] - want).abs() <= off).all()
    assert (rstd[0, 1] - r).abs() <= 36 * ref.U * 5 * r


@pytest.mark.parametrize("rows", [3, 80])
def test_gelu_on_its_flat_side(layers, rows):  # noqa: F811
    """g from -2 to -9, where 1 + erf(g / sqrt 2) has lost its digits and erfc(-g / sqrt 2) has not: that is off by a few
    roundings, and by 2 t^2 = g^2 times the two of its argument t."""
    n, width, hidden = 1, 33, 40
    gate, up, down = torch.zeros(n, hidden, width), torch.zeros(n, hidden, width), torch.zeros(n, width, hidden)
    g = -torch.linspace(2.0, 9.0, width)
    gate[0, 0], up[0, 0], down[0, :, 0] = g, 1.0, 1.0
    x = torch.eye(width).repeat(1, (rows + width - 1) // width, 1)[:, :rows]
    d = g.double()[torch.arange(rows) % width]
    h = d * 0.5 * torch.special.erfc(-d / math.sqrt(2))
    y, _ = layers.gated_ffn_forward(x.cuda(), gate.cuda(), up.cuda(), down.cuda(), "gelu")
    want = h[None, :, None].expand(n, rows, width)
    ref.check(y, (want, (32 + 2 * d * d)[None, :, None] * ref.U * want.abs()), "y")
