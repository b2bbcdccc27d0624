"""The particles' layers in 64 bits, straight from their definitions, and how far fp32 arithmetic may be from them: running error
bounds, value by value.  A sum of K products in fp32 is off by at most K + 6 roundings of 2^-24 of the sum of their
absolute values (what a product leaves out of its operands' parts is below two more); what is computed from inexact values carries their
bounds along, to first order."""
import math

import torch

U = 2.0 ** -24  # half a step of fp32


def rounding(dtype):
    return torch.finfo(dtype).eps / 2


def activation(g, name):
    """act, act' and bounds on |act'| and |act''|"""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), 1.1, 0.5
    cdf = 0.5 * (1 + torch.special.erf(g / math.sqrt(2)))
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 1.13, 0.8


def product(a, ea, b, eb, extra=0.0):
    """a b^T over the last dimensions, with its bound; `extra`: what is left out of the operands on purpose."""
    k = a.shape[-1]
    bt, at = b.transpose(-1, -2).abs(), a.abs()
    bound = ((k + 8) * U + extra) * (at @ bt)
    if ea is not None:
        bound = bound + ea @ bt
    if eb is not None:
        bound = bound + at @ eb.transpose(-1, -2)
    return a @ b.transpose(-1, -2), bound


def gated_ffn(x, gate, up, down, act, dy=None):
    """{name: (value, bound)} of y and, with dy, of the gradients.  Inputs as the kernels get them."""
    half = x.dtype != torch.float32
    left_out = 2.0 ** -15 if half else 0.0  # two parts of each operand where the result has 16 bits
    r = rounding(x.dtype)
    x, gate, up, down = (t.double().cpu() for t in (x, gate, up, down))
    g, eg = product(x, None, gate, None)
    u, eu = product(x, None, up, None)
    a, slope, s1, s2 = activation(g, act)
    ea = s1 * eg + 8 * U * g.abs()
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + 2 * U * h.abs()
    y, ey = product(h, eh, down, None, left_out)
    out = {"y": (y, ey + r * y.abs())}
    if dy is None:
        return out
    dy = dy.double().cpu()
    dh, edh = product(dy, None, down.transpose(1, 2), None)
    dg, du = dh * u * slope, dh * a
    edg = edh * (u * slope).abs() + dh.abs() * (eu * slope.abs() + u.abs() * (s2 * eg + 8 * U * (1 + g.abs()))) + 3 * U * dg.abs()
    edu = edh * a.abs() + dh.abs() * ea + 2 * U * du.abs()
    d1, e1 = product(dg, edg, gate.transpose(1, 2), None, left_out)
    d2, e2 = product(du, edu, up.transpose(1, 2), None, left_out)
    # one sum over both: as many roundings more
    dx, edx = d1 + d2, e1 + e2 + gate.shape[1] * U * (dg.abs() @ gate.abs() + du.abs() @ up.abs())
    out["dx"] = (dx, edx + r * dx.abs())
    for name, d, e in (("dgate", dg, edg), ("dup", du, edu)):
        v, b = product(d.transpose(1, 2), e.transpose(1, 2), x.transpose(1, 2), None)
        out[name] = (v, b + U * v.abs())
    v, b = product(dy.transpose(1, 2), None, h.transpose(1, 2), eh.transpose(1, 2))
    out["ddown"] = (v, b + U * v.abs())
    return out


def layer_norm(x, weight, bias, eps, dy=None):
    r = rounding(x.dtype)
    x, weight = x.double().cpu(), weight.double().cpu()[:, None]
    bias = torch.zeros_like(weight) if bias is None else bias.double().cpu()[:, None]
    d = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    emean = (d + 1) * U * x.abs().mean(-1, keepdim=True)
    c = x - mean
    ec = emean + U * c.abs()
    var = (c * c).mean(-1, keepdim=True)
    # (sum c = 0: an error of the mean enters the variance squared)
    evar = (d + 4) * U * var + emean ** 2 + 2 * U * (c.abs() * c.abs()).mean(-1, keepdim=True)
    rstd = (var + eps).rsqrt()
    erel = evar / (2 * (var + eps)) + 3 * U
    xhat = c * rstd
    exh = ec * rstd + xhat.abs() * (erel + 2 * U)
    y = xhat * weight + bias
    ey = exh * weight.abs() + 2 * U * ((xhat * weight).abs() + y.abs())
    out = {"y": (y, ey + r * y.abs()), "mean": (mean[..., 0], emean[..., 0]), "rstd": (rstd[..., 0], (rstd * erel)[..., 0] + U * rstd[..., 0])}
    if dy is None:
        return out
    dy = dy.double().cpu()
    a = dy * weight
    ea = U * a.abs()
    ma, max_ = a.mean(-1, keepdim=True), (a * xhat).mean(-1, keepdim=True)
    ema = (ea + (d + 1) * U * a.abs()).mean(-1, keepdim=True)
    emax = (ea * xhat.abs() + a.abs() * exh + (d + 2) * U * (a * xhat).abs()).mean(-1, keepdim=True)
    t = a - ma - xhat * max_
    et = ea + ema + exh * max_.abs() + xhat.abs() * emax + 4 * U * (a.abs() + ma.abs() + (xhat * max_).abs())
    dx = rstd * t
    edx = rstd * et + dx.abs() * (erel + 2 * U)
    out["dx"] = (dx, edx + r * dx.abs())
    rows = x.shape[1]
    out["dweight"] = ((dy * xhat).sum(1), (dy.abs() * exh + (rows + 2) * U * (dy * xhat).abs()).sum(1))
    out["dbias"] = (dy.sum(1), ((rows + 2) * U * dy.abs()).sum(1))
    return out


_M64 = (1 << 64) - 1


def splitmix64(v):
    z = (v + 0x9E3779B97F4A7C15) & _M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & _M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & _M64
    return z ^ (z >> 31)


def kept(size, p, seed, call, counter=None, start=0):
    """Which of the values start .. start + size - 1 dropout keeps, in Python integers."""
    base = splitmix64((splitmix64(seed & _M64) + call) & _M64)
    if counter is not None:
        base = splitmix64((base + counter) & _M64)
    limit = round(p * 2 ** 32)
    out = []
    for e in range(start, start + size):
        h = splitmix64((base + e // 2) & _M64)
        out.append((h & 0xFFFFFFFF if e % 2 else h >> 32) >= limit)
    return torch.tensor(out, dtype=torch.bool)


def check(got, ref, what):
    """Every value within its bound (and a denormal of the type)."""
    value, bound = ref
    got = got.double().cpu()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    off = (got - value).abs() - bound
    assert not torch.isnan(off).any(), f"{what}: NaN"
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 1e-37, f"{what}: {worst:.3e} beyond its bound at {torch.nonzero(off == off.max())[0].tolist()}"
