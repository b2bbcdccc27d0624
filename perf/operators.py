"""What is timed when the speed of the particles' own layers is looked at: layer norm, gated feed-forward block
and dropout of n networks at once, their parameters rows of one (n, D) float32 matrix X as the all-particle update
takes it, the gradients of the parameters written to the same places of a matrix G.

A case is a dict: `op` ("norm", "ffn", "dropout"), `pass` ("forward": what prediction runs; "train": forward
and backward), `type` of the activations ("float32", "bfloat16", "float16"; parameters and their gradients are
float32), `n` particles with `rows` rows of `width` values each, and
    offset   where the layer's parameters start in a row of X: behind those of earlier layers (norm, ffn)
    hidden   width of the hidden layer, `act` its activation (ffn)
    p        probability of dropping a value, `residual` whether the result is added to a residual stream (dropout)

With `own` false the operators are computed by plain torch operations in 32 bits and rounded once.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_MASK32 = 0xFFFFFFFF
_GAMMA, _MUL1, _MUL2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB  # splitmix64


def listed():
    def norm(name, way, kind, n, rows, width, offset):
        return {"name": name, "op": "norm", "pass": way, "type": kind, "n": n, "rows": rows, "width": width, "offset": offset}

    def ffn(name, way, kind, n, rows, width, hidden, act, offset):
        return {"name": name, "op": "ffn", "pass": way, "type": kind, "n": n, "rows": rows, "width": width, "hidden": hidden,
                "act": act, "offset": offset}

    def dropout(name, way, kind, n, rows, width, p, residual):
        return {"name": name, "op": "dropout", "pass": way, "type": kind, "n": n, "rows": rows, "width": width, "p": p,
                "residual": residual}

    return [
        # one input to sixteen small networks: nothing but latency
        norm("norm_token", "forward", "float32", 16, 1, 64, 0),
        # eight small vision networks, a minibatch of eight images of 197 patches
        norm("norm_train", "train", "bfloat16", 8, 8 * 197, 384, 0),
        # odd everything, parameters off the 16-byte boundaries
        norm("norm_odd_train", "train", "float32", 5, 1_003, 1_001, 8_577),
        # the widest stream that the largest ensembles normalise
        norm("norm_large_train", "train", "bfloat16", 16, 8_192, 1_024, 0),
        # the predictive mean of sixteen networks for one input
        ffn("ffn_token", "forward", "float32", 16, 1, 256, 683, "silu", 0),
        # a handful of inputs to eight large networks
        ffn("ffn_few_rows", "forward", "bfloat16", 8, 5, 1_024, 2_731, "silu", 2_048),
        # a full-batch step of sixteen small networks, width of the PINN-sized MLPs
        ffn("ffn_small_train", "train", "float32", 16, 200, 64, 171, "gelu", 129),
        # eight small vision networks as above
        ffn("ffn_train", "train", "float32", 8, 8 * 197, 384, 1_024, "silu", 768),
        # eight large networks in mixed precision
        ffn("ffn_large_train", "train", "bfloat16", 8, 4_096, 1_024, 2_730, "silu", 2_048),
        # dropout kept on in prediction, small networks
        dropout("dropout_small", "forward", "float32", 4, 16, 64, 0.1, False),
        # odd sizes, half precision
        dropout("dropout_odd_train", "train", "float16", 7, 999, 333, 0.25, False),
        # the residual stream of the largest ensembles
        dropout("dropout_large_train", "train", "bfloat16", 16, 8_192, 1_024, 0.1, True),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e14)


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "ffn", "ffn", "dropout"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        c = {"op": op, "pass": rng.choice(["forward", "train"]), "type": rng.choice(list(_TYPES)), "n": _log_between(rng, 1, 64),
             "rows": _log_between(rng, 1, 16_384)}
        if op == "ffn":
            c["width"] = _log_between(rng, 16, 1_536)
            c["hidden"] = int(c["width"] * rng.uniform(1.5, 4.5))
            if rng.random() < 0.5:
                c["width"], c["hidden"] = max(32, c["width"] // 32 * 32), max(32, c["hidden"] // 32 * 32)
            c["act"] = rng.choice(["silu", "gelu"])
        else:
            c["width"] = _log_between(rng, 8, 8_192)
            if rng.random() < 0.5:
                c["width"] = max(32, c["width"] // 32 * 32)
        if op == "dropout":
            c["p"], c["residual"] = rng.choice([0.0, 0.1, 0.25, 0.5, rng.random()]), rng.random() < 0.5
        else:
            c["offset"] = rng.choice([0, 32 * rng.randint(1, 100), rng.randint(1, 10_000)])
        if _cost(c) <= most and 3072 not in (c["rows"], c["width"], c.get("hidden")):
            return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _layers(matrix, case):
    """The layer's parameters (or their gradients), views into the rows of X (or G)."""
    n, d, at = case["n"], case["width"], case["offset"]
    shapes = [(d,), (d,)] if case["op"] == "norm" else [(case["hidden"], d), (case["hidden"], d), (d, case["hidden"])]
    views = []
    for shape in shapes:
        size = math.prod(shape)
        views.append(matrix[:, at:at + size].view(n, *shape))
        at += size
    return views


def _params(case):
    d = case["width"]
    return case["offset"] + (2 * d if case["op"] == "norm" else 3 * d * case["hidden"])


def _rows_matrix(n, D):
    """An (n, D) view whose rows start on 128-byte boundaries, as the update likes them best."""
    return torch.zeros(n, (D + 31) // 32 * 32, device="cuda")[:, :D]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, t, d, kind = case["n"], case["rows"], case["width"], _TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    state = {"case": case}
    if case["op"] == "norm":  # a residual stream: its rows are off centre and of different lengths
        state["x"] = (normal(n, t, d) * (0.5 + normal(n, t, 1).abs()) + 0.5 * normal(n, t, 1)).to(kind)
    else:
        state["x"] = normal(n, t, d).to(kind)
    if case["pass"] == "train":
        state["dy"] = (normal(n, t, d) * 1e-2).to(kind)
    if case["op"] == "dropout":
        state["seed"], state["call"] = seed + 230_606_528, 3
        if case["residual"]:
            state["residual"] = normal(n, t, d).to(kind)
        return state
    D = _params(case)
    X, G = _rows_matrix(n, D), _rows_matrix(n, D)
    views = _layers(X, case)
    if case["op"] == "norm":
        views[0].copy_(1.0 + 0.1 * normal(n, d))
        views[1].copy_(0.1 * normal(n, d))
    else:
        for v in views:
            v.copy_(normal(*v.shape) * v.shape[-1] ** -0.5)
    state["X"], state["G"] = X, G
    state["params"], state["grads"] = views, _layers(G, case)
    return state


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _norm_plain(state, train):
    case, x = state["case"], state["x"].float()
    weight, bias = state["params"]
    mean = x.mean(-1, keepdim=True)
    centred = x - mean
    rstd = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    xhat = centred * rstd
    out = {"y": (xhat * weight[:, None] + bias[:, None]).to(_TYPES[case["type"]])}
    if train:
        dy = state["dy"].float()
        a = dy * weight[:, None]
        dx = rstd * (a - a.mean(-1, keepdim=True) - xhat * (a * xhat).mean(-1, keepdim=True))
        out |= {"dx": dx.to(_TYPES[case["type"]]), "dweight": (dy * xhat).sum(1), "dbias": dy.sum(1)}
    return out


def _activation(g, act):
    """The activation and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    cdf = 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5


def _ffn_plain(state, train):
    case, x = state["case"], state["x"].float()
    kind = _TYPES[case["type"]]
    gate, up, down = state["params"]
    g, u = x @ gate.transpose(1, 2), x @ up.transpose(1, 2)
    a, da = _activation(g, case["act"])
    h = a * u
    out = {"y": (h @ down.transpose(1, 2)).to(kind)}
    if train:
        dy = state["dy"].float()
        dh = dy @ down
        dg, du = dh * u * da, dh * a
        out |= {"dx": (dg @ gate + du @ up).to(kind), "dgate": dg.transpose(1, 2) @ x, "dup": du.transpose(1, 2) @ x,
                "ddown": dy.transpose(1, 2) @ h}
    return out


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _shift(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)


def _mix(z):
    """splitmix64's output function on int64 bit patterns."""
    z = (z ^ _shift(z, 30)) * _signed(_MUL1)
    z = (z ^ _shift(z, 27)) * _signed(_MUL2)
    return z ^ _shift(z, 31)


def _stream(seed, call):
    def mix(v):
        v = (v + _GAMMA) & ((1 << 64) - 1)
        v = ((v ^ (v >> 30)) * _MUL1) & ((1 << 64) - 1)
        v = ((v ^ (v >> 27)) * _MUL2) & ((1 << 64) - 1)
        return v ^ (v >> 31)
    return mix((mix(seed) + call) & ((1 << 64) - 1))


def _dropout_plain(state, train):
    case, x = state["case"], state["x"]
    kind, p, size = _TYPES[case["type"]], case["p"], x.numel()
    # value e is kept if the (e mod 2)-th half of the stream's hash e / 2, upper half first, is not below p 2^32
    z = _mix(torch.arange((size + 1) // 2, device=x.device) + _signed(_stream(state["seed"], state["call"]) + _GAMMA))
    u = torch.stack([_shift(z, 32), z & _MASK32], 1).reshape(-1)[:size].view(x.shape)
    keep = u >= round(p * 4294967296.0)
    scale = 1.0 / (1.0 - p)
    y = torch.where(keep, x.float() * scale, 0.0)
    if case["residual"]:
        y = y + state["residual"].float()
    out = {"y": y.to(kind)}
    if train:
        out["dx"] = torch.where(keep, state["dy"].float() * scale, 0.0).to(kind)
    return out


def run(state):
    case, train = state["case"], state["case"]["pass"] == "train"
    op = case["op"]
    if not own:
        return {"norm": _norm_plain, "ffn": _ffn_plain, "dropout": _dropout_plain}[op](state, train)
    from paper_2306_06528_amd import layers
    if op == "norm":
        (weight, bias), (dweight, dbias) = state["params"], state["grads"]
        y, mean, rstd = layers.layer_norm_forward(state["x"], weight, bias, EPS)
        if not train:
            return {"y": y}
        dx = layers.layer_norm_backward(state["dy"], state["x"], weight, mean, rstd, dweight, dbias)
        return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "ffn":
        (gate, up, down), (dgate, dup, ddown) = state["params"], state["grads"]
        y, saved = layers.gated_ffn_forward(state["x"], gate, up, down, case["act"], save=train)
        if not train:
            return {"y": y}
        dx = layers.gated_ffn_backward(state["dy"], state["x"], gate, up, down, saved, dgate, dup, ddown, case["act"])
        return {"y": y, "dx": dx, "dgate": dgate, "dup": dup, "ddown": ddown}
    y = layers.dropout_forward(state["x"], case["p"], state["seed"], state["call"], state.get("residual"))
    if not train:
        return {"y": y}
    return {"y": y, "dx": layers.dropout_backward(state["dy"], case["p"], state["seed"], state["call"])}


def work(case):
    n, t, d = case["n"], case["rows"], case["width"]
    size = {"float32": 4, "bfloat16": 2, "float16": 2}[case["type"]]
    train = case["pass"] == "train"
    acts = size * n * t * d * (4 if train else 2)  # x and y, dy and dx
    if case["op"] == "norm":
        return {"bytes": acts + 4 * n * 2 * d * (2 if train else 1), "flops": n * t * d * (19 if train else 7)}
    if case["op"] == "ffn":
        f = case["hidden"]
        return {"bytes": acts + 4 * n * 3 * d * f * (2 if train else 1), "flops": 6 * n * t * d * f * (3 if train else 1)}
    return {"bytes": acts + (size * n * t * d if case["residual"] else 0), "flops": n * t * d * (16 if train else 9)}


# ---------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_norm(state, i):
    x, (w, b) = state["x"][i].double(), (v[i].double() for v in state["params"])
    sigma = torch.sqrt(x.var(-1, unbiased=False) + EPS)[:, None]
    xhat = (x - x.mean(-1)[:, None]) / sigma
    out = {"y": xhat * w + b}
    if "dy" in state:
        dy = state["dy"][i].double()
        dxhat = dy * w
        d = x.shape[-1]
        out["dx"] = (d * dxhat - dxhat.sum(-1)[:, None] - xhat * (dxhat * xhat).sum(-1)[:, None]) / (d * sigma)
        out["dweight"], out["dbias"] = torch.einsum("td,td->d", dy, xhat), dy.sum(0)
    return out


def _exact_ffn(state, i):
    x, (gate, up, down) = state["x"][i].double(), (v[i].double() for v in state["params"])
    g, u = torch.mm(x, gate.t()), torch.mm(x, up.t())
    if state["case"]["act"] == "silu":
        s = torch.sigmoid(g)
        a, slope = g * s, s + g * s * (1 - s)
    else:
        s = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        a, slope = g * s, s + g * torch.exp(-g.square() / 2) / math.sqrt(2.0 * math.pi)
    out = {"y": torch.mm(a * u, down.t())}
    if "dy" in state:
        dy = state["dy"][i].double()
        dh = torch.mm(dy, down)
        out["dx"] = torch.mm(dh * u * slope, gate) + torch.mm(dh * a, up)
        out["dgate"], out["dup"] = torch.mm((dh * u * slope).t(), x), torch.mm((dh * a).t(), x)
        out["ddown"] = torch.mm(dy.t(), a * u)
    return out


def _exact_keep(case, state):
    """Which values are kept, by unsigned arithmetic on the host."""
    size = case["n"] * case["rows"] * case["width"]
    base = np.uint64(_stream(state["seed"], state["call"]))
    keep = np.empty((size + 1) // 2 * 2, dtype=bool)
    limit = round(case["p"] * 2.0 ** 32)
    for start in range(0, keep.size // 2, 1 << 20):
        z = np.arange(start, min(start + (1 << 20), keep.size // 2), dtype=np.uint64) + base + np.uint64(_GAMMA)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(_MUL1)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(_MUL2)
        z ^= z >> np.uint64(31)
        keep[2 * start:2 * (start + z.size):2] = (z >> np.uint64(32)) >= np.uint64(limit)
        keep[2 * start + 1:2 * (start + z.size):2] = (z & np.uint64(_MASK32)) >= np.uint64(limit)
    return torch.from_numpy(keep[:size]).cuda().view(case["n"], case["rows"], case["width"])


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "dropout":
        drop = ~_exact_keep(case, state)
        parts = {"y": (state["x"].double() / (1.0 - case["p"])).masked_fill(drop, 0.0)}
        if case["residual"]:
            parts["y"] += state["residual"].double()
        if case["pass"] == "train":
            parts["dx"] = (state["dy"].double() / (1.0 - case["p"])).masked_fill(drop, 0.0)
        return parts
    one = _exact_norm if case["op"] == "norm" else _exact_ffn
    each = [one(state, i) for i in range(case["n"])]
    return {k: torch.stack([e[k] for e in each]) for k in each[0]}
