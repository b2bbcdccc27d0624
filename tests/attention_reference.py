"""The attention half of the particles' layers in 64 bits, straight from the definitions, and how far the kernels may be from them: running error
bounds, value by value, as layer_reference.py has them.  U is half a step of fp32, r half a step of the activations' type.

What the kernels round on the way, besides fp32 sums: probabilities to the activations' type for their product with the values (r of each; fp16 holds
them 2^6 times as large relative to a maximum that is at most 2^8 too low, so what falls below its smallest step is below 2^-25 2^-6 of the largest probability, and 2^-25 2^-14 of 1 in the
backward pass), the gradients of scores for their products with keys and queries (r of each; fp16 ones scaled so that the largest so far is 2^13 at
least: 2^-25 2^-13 of the largest), and o, from which the backward pass makes delta."""
import math

import torch

from layer_reference import U, check, product, rounding  # noqa: F401

FLOOR = {torch.float32: (0.0, 0.0, 0.0), torch.bfloat16: (0.0, 0.0, 0.0), torch.float16: (2.0 ** -31, 2.0 ** -39, 2.0 ** -38)}


def stored(value, dtype):
    """What rounding a value for its output is off by at most: half a step, r of the value, but of fp16 values below 2^-14, whose steps are 2^-24 whatever their
    size, 2^-25 (bf16 and fp32 have these steps below 1e-38)."""
    return (rounding(dtype) * value.abs()).clamp(min=2.0 ** -25 if dtype == torch.float16 else 0.0)


def cpu64(*ts):
    return [None if t is None else t.detach().double().cpu() for t in ts]


# ---------------------------------------------------------------------------------------------
# linear map
# ---------------------------------------------------------------------------------------------
def activation(z, name):
    """act, act' and bounds on |act'| and |act''|"""
    if name == "none":
        return z, torch.ones_like(z), 1.0, 0.0
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), 1.0, 0.0
    if name == "tanh":
        t = torch.tanh(z)
        return t, 1 - t * t, 1.0, 0.77
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s)), 1.1, 0.5
    cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 1.13, 0.8


def linear(x, weight, bias, act, residual=None, dy=None):
    """{name: (value, bound)}.  relu's step: where z is within its bound of 0 either side is right, so those gradients have bounds as large as themselves."""
    kind = x.dtype
    x, weight, bias, residual, dy = cpu64(x, weight, bias, residual, dy)
    z, ez = product(x, None, weight, None)
    if bias is not None:
        z = z + bias[:, None]
        ez = ez + U * z.abs()
    a, slope, s1, s2 = activation(z, act)
    y, ey = a, s1 * ez + 8 * U * a.abs() + (0 if act in ("none", "relu") else 2 * U * z.abs() * (a != 0))
    if residual is not None:
        y = y + residual
        ey = ey + U * y.abs()
    out = {"y": (y, ey + stored(y, kind))}
    if dy is None:
        return out
    dz = dy * slope
    edz = dy.abs() * (s2 * ez + (0 if act == "none" else 10 * U * (1 + z.abs()) * (act != "relu")))
    if act == "relu":
        edz = torch.where(z.abs() <= ez, dy.abs(), edz)
    if act == "none":
        edz = None
    dx, edx = product(dz, edz, weight.transpose(1, 2), None)
    out["dx"] = (dx, edx + stored(dx, kind))
    v, e = product(dz.transpose(1, 2), None if edz is None else edz.transpose(1, 2), x.transpose(1, 2), None)
    out["dweight"] = (v, e + U * v.abs())
    rows = x.shape[1]
    out["dbias"] = (dz.sum(1), ((rows + 4) * U * dz.abs() + (0 if edz is None else edz)).sum(1))
    return out


# ---------------------------------------------------------------------------------------------
# norms and rotation
# ---------------------------------------------------------------------------------------------
def turned(x, angle, layout, back=False):
    """The first 2 * angle.shape[-1] values of the last dimension turned; angle broadcasts over the rest."""
    p = angle.shape[-1]
    if p == 0:
        return x
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if back else 1)
    out = x.clone()
    i, j = (slice(0, p), slice(p, 2 * p)) if layout == "half" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    out[..., i] = x[..., i] * c - x[..., j] * s
    out[..., j] = x[..., j] * c + x[..., i] * s
    return out


def around(x, p, layout):
    """What a turned value is made of, at most: |a| + |b| of its pair."""
    out = x.abs().clone()
    if p:
        i, j = (slice(0, p), slice(p, 2 * p)) if layout == "half" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
        out[..., i] = out[..., j] = x[..., i].abs() + x[..., j].abs()
    return out


def qk_norm_rotary(x, weight, frequencies, positions, layout, eps, dy=None):
    """One of q and k, (n, batch, tokens, heads, dim): {"y", "dx", "dweight"}"""
    kind, dim = x.dtype, x.shape[-1]
    x, weight, frequencies, dy = cpu64(x, weight, frequencies, dy)
    if frequencies is None:
        angle = torch.zeros(1, 0, dtype=torch.float64)
        far = torch.zeros(())
    else:
        positions = positions.cpu().double()
        angle = (positions[..., None] * frequencies)[..., None, :]  # (batch or none, tokens, 1, pairs)
        far = angle.abs().max() * 2.0 ** -51 if angle.numel() else torch.zeros(())
    p = angle.shape[-1]
    et = 8 * U + far  # of cos and sin, the sum of two products
    if weight is None:
        y = turned(x, angle, layout)
        out = {"y": (y, (et if p else 0.0) * around(x, p, layout) + stored(y, kind))}
        if dy is not None:
            dx = turned(dy, angle, layout, True)
            out["dx"] = (dx, (et if p else 0.0) * around(dy, p, layout) + stored(dx, kind))
        return out
    w = weight[:, None, None, None]
    square = (x * x).mean(-1, keepdim=True)
    rstd = (square + eps).rsqrt()
    er = (dim + 8) * U  # relative
    xhat = x * rstd
    v = xhat * w
    y = turned(v, angle, layout)
    out = {"y": (y, (er + 4 * U + (et if p else 0.0)) * around(v, p, layout) + stored(y, kind))}
    if dy is None:
        return out
    g = turned(dy, angle, layout, True)
    eg = (et if p else 0.0) * around(dy, p, layout)
    a, ea = g * w, eg * w.abs() + U * (g * w).abs()
    m = (a * xhat).mean(-1, keepdim=True)
    em = (ea * xhat.abs() + (er + (dim + 6) * U) * (a * xhat).abs()).mean(-1, keepdim=True)
    dx = rstd * (a - xhat * m)
    edx = rstd * (ea + xhat.abs() * em + (2 * er + 4 * U) * (a.abs() + (xhat * m).abs())) + er * dx.abs()
    out["dx"] = (dx, edx + stored(dx, kind))
    count = x[0, ..., 0].numel()
    out["dweight"] = ((g * xhat).sum((1, 2, 3)), (eg * xhat.abs() + (er + (count + 6) * U) * (g * xhat).abs()).sum((1, 2, 3)))
    return out


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------
def seen(batch, t, s, causal=False, starts=None, lengths=None, documents=None, prefix=None):
    """(batch, t, s): which key a query sees, straight from the rule; and the distances."""
    see = torch.zeros(batch, t, s, dtype=torch.bool)
    far = torch.zeros(batch, t, s, dtype=torch.float64)
    j = torch.arange(s)
    for b in range(batch):
        first = s - t if starts is None else int(starts[b])
        for i in range(t):
            p = first + i
            far[b, i] = (p - j).abs().double()
            ok = j < (s if lengths is None else int(lengths[b]))
            if causal:
                ok &= (j <= p) | (j < (0 if prefix is None else int(prefix[b])))
            if documents is not None:
                ok &= (documents[b].cpu() == documents[b, p].cpu()) if 0 <= p < s else torch.zeros(s, dtype=torch.bool)
            see[b, i] = ok
    return see, far


def attention(q, k, v, do=None, causal=False, cap=0.0, slopes=None, scale=None, starts=None, lengths=None, documents=None, prefix=None):
    """{name: (value, bound)} of o, lse and, with do, of the gradients.  Values that nobody sees may be anything: they are taken as 0."""
    kind = q.dtype
    r = rounding(kind) if kind != torch.float32 else 0.0
    low_p, low_pb, low_z = FLOOR[kind]
    n, batch, t, heads, d = q.shape
    s, kv = k.shape[2], k.shape[3]
    scale = d ** -0.5 if scale is None else scale
    see, far = seen(batch, t, s, causal, starts, lengths, documents, prefix)
    if lengths is not None:
        hidden = torch.arange(s)[None] >= lengths.cpu()[:, None].long()  # (batch, s): never read
        k, v = (torch.where(hidden[None, :, :, None, None].to(x.device), torch.zeros((), dtype=x.dtype, device=x.device), x) for x in (k, v))
    q, k, v, do, slopes = cpu64(q, k, v, do, slopes)
    group = heads // kv

    def split(x, per):  # (n, batch, kv, per, tokens, d)
        return x.reshape(*x.shape[:3], kv, per, d).permute(0, 1, 3, 4, 2, 5)

    def joined(x):
        return x.permute(0, 1, 4, 2, 3, 5).flatten(3, 4)
    Q, K, V = split(q, group), split(k, 1), split(v, 1)
    see, far = see[None, :, None, None], far[None, :, None, None]
    z = scale * (Q @ K.transpose(-1, -2))
    ez = scale * (d + 8) * U * (Q.abs() @ K.abs().transpose(-1, -2)) + 3 * U * z.abs()
    damp, edamp = 1.0, 0.0
    if cap:
        th = torch.tanh(z / cap)
        damp = 1 - th * th
        edamp = 0.8 / cap * ez + 12 * U
        z = cap * th
        ez = ez * damp.clamp(min=0) + ez * ez / cap + 8 * U * cap
    if slopes is not None:
        sl = slopes.reshape(n, 1, kv, group, 1, 1)
        ez = ez + 4 * U * (sl * far).abs()
        z = z - sl * far
        ez = ez + 2 * U * z.abs()
    z = z.masked_fill(~see, -math.inf)
    none = ~see.any(-1, keepdim=True)
    lse = torch.logsumexp(z, -1, keepdim=True)
    P = torch.exp(z - lse).masked_fill(~see, 0.0).masked_fill(none, 0.0)
    safe = torch.where(none, 0.0, lse)
    big = torch.where(see, z.abs(), 0.0).amax(-1, keepdim=True) if s else torch.zeros_like(safe)
    rel = torch.where(see, ez + 8 * U * (1 + z.abs() + big), 0.0)  # of exp z
    total = (P * rel).sum(-1, keepdim=True) + (s + 8) * U  # of their sum
    el = total + 4 * U * (1 + safe.abs() + big)
    o = P @ V
    eP = P * (rel + total + r) + low_p * see
    eo = eP @ V.abs() + (s + 16) * U * (P @ V.abs()) + stored(o, kind)
    out = {"o": (joined(o), joined(eo))}
    L = lse.squeeze(-1).flatten(2, 3)
    out["lse"] = (L, torch.where(torch.isinf(L), 0.0, el.expand_as(lse).squeeze(-1).flatten(2, 3)))
    if do is None:
        return out
    D = split(do, group)
    dp = D @ V.transpose(-1, -2)
    edp = (d + 8) * U * (D.abs() @ V.abs().transpose(-1, -2))
    delta = (D * o).sum(-1, keepdim=True)
    edelta = (D.abs() * eo).sum(-1, keepdim=True) + (d + 8) * U * (D * o).abs().sum(-1, keepdim=True)
    rp = rel + el + 4 * U  # of P made again
    dz = P * (dp - delta)
    e0 = rp * (dz.abs() + P * edelta) + P * (edp + 2 * U * (dp.abs() + delta.abs() + edelta))
    edz = e0 + P * edelta
    if slopes is not None:  # what delta's error puts on a row's sum is taken off again, with the row's mean distance
        mean = (P * far).sum(-1, keepdim=True)
        value = -(dz * far).sum((1, 4, 5)).reshape(n, heads)
        bound = (e0 * (far + mean) + (rp + total) * P * edelta * (far + mean) + (s + t * batch + 16) * U * (dz.abs() + P * edelta) * (far + mean)).sum((1, 4, 5)).reshape(n, heads)
        out["dslopes"] = (value, bound)
    if cap:
        edz = edz * damp + dz.abs() * edamp + edz * edamp
        dz = dz * damp
    most = dz.abs().amax((-1, -2), keepdim=True) if s and t else torch.zeros(())
    ez16 = edz + r * (dz.abs() + edz) + low_z * (most + edz) * see
    dq = scale * (dz @ K)
    edq = scale * (ez16 @ K.abs() + (s + 16) * U * (dz.abs() + ez16) @ K.abs()) + stored(dq, kind)
    out["dq"] = (joined(dq), joined(edq))
    rows = t * group
    dzt, ezt = dz.transpose(-1, -2), ez16.transpose(-1, -2)
    dk = scale * (dzt @ Q).sum(3, keepdim=True)
    edk = scale * (ezt @ Q.abs() + (rows + 16) * U * (dzt.abs() + ezt) @ Q.abs()).sum(3, keepdim=True) + stored(dk, kind)
    out["dk"] = (joined(dk), joined(edk))
    Pt, ePt = P.transpose(-1, -2), (P * (rp + r) + low_pb * see).transpose(-1, -2)
    dv = (Pt @ D).sum(3, keepdim=True)
    edv = (ePt @ D.abs() + (rows + 16) * U * Pt @ D.abs()).sum(3, keepdim=True) + stored(dv, kind)
    out["dv"] = (joined(dv), joined(edv))
    return out


def check_lse(got, ref):
    """Rows that see nothing are -infinity in both."""
    value, bound = ref
    got = got.double().cpu()
    assert torch.equal(torch.isinf(got), torch.isinf(value))
    inf = torch.isinf(value)
    check(torch.where(inf, 0.0, got), (torch.where(inf, 0.0, value), bound), "lse")
