"""What is timed when the speed of the attention half of the particles' layers is looked at: linear maps with bias, activation and
residual, norms of queries and keys with the rotation by their positions, and attention, of n networks at once.  As in the rest of the
package the networks' parameters are rows of one (n, D) float32 matrix X and their gradients go to the same places of a matrix G.

A case is a dict: `op` ("linear", "rotary", "attention"), `pass` ("forward": what prediction runs; "train": forward and backward),
`type` of the activations ("float32", "bfloat16", "float16"; parameters and their gradients are float32), `n` particles, `offset` where the
operator's parameters start in a row of X, and

    linear     y = act(x weight^T + bias) + residual for `rows` rows of `width` values, `out` of them in a result; `act` "none", "silu", "gelu",
               "relu" or "tanh", `residual` whether one is added
    rotary     q of `heads` and k of `kv_heads` heads of `dim` values, `batch` sequences of `length` tokens each; `norm` whether every head is
               divided by its root mean square and multiplied by a weight; the first `rotary` values of a head are rotated (0: none), `layout`
               "half" or "interleaved", `scaling` "none", "linear" or "parts" (wavelengths longer than the trained context are stretched, short
               ones stay), `start` the first token's position; `fused`: q and k are views into the results of one linear map
    attention  `batch` sequences, `length` queries and `keys` keys each, `heads` over `kv_heads` heads of `dim` values; `causal`; `cap` (0: none) of
               the scores, by tanh; `bias` whether a slope per head times the distance is taken off the scores; `prefix` keys that every query
               sees (causal); `documents`: sequences are so many documents that do not see one another (0: one);
               `ragged`: the sequences' keys end at different places (a cache that was filled so far, its queries the last tokens)

With `own` false the operators are computed by plain torch operations in 32 bits (angles in 64) and rounded once.
"""
import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10_000.0
TRAINED = 2_048  # tokens: the context that scaled rotations are scaled from
FACTOR = 8.0
_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    def linear(name, way, kind, n, rows, width, out, act, residual, offset):
        return {"name": name, "op": "linear", "pass": way, "type": kind, "n": n, "rows": rows, "width": width, "out": out, "act": act,
                "residual": residual, "offset": offset}

    def rotary(name, way, kind, n, batch, length, heads, kv_heads, dim, turned, layout, scaling, start, offset):
        return {"name": name, "op": "rotary", "pass": way, "type": kind, "n": n, "batch": batch, "length": length, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "norm": True, "rotary": turned, "layout": layout, "scaling": scaling, "start": start,
                "fused": True, "offset": offset}

    def attention(name, way, kind, n, batch, length, keys, heads, kv_heads, dim, causal=False, cap=0.0, bias=False, prefix=0, documents=0,
                  ragged=False):
        return {"name": name, "op": "attention", "pass": way, "type": kind, "n": n, "batch": batch, "length": length, "keys": keys, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "causal": causal, "cap": cap, "bias": bias, "prefix": prefix, "documents": documents,
                "ragged": ragged, "offset": 0}

    return [
        # q, k and v of one input to sixteen small networks: nothing but latency
        linear("linear_token", "forward", "float32", 16, 1, 256, 768, "none", False, 0),
        # the hidden layer of small regression networks, a full batch of odd size
        linear("linear_odd_train", "train", "float32", 5, 1_003, 333, 501, "tanh", False, 129),
        # eight vision networks, a minibatch of eight images of 197 patches: back into the residual stream
        linear("linear_large_train", "train", "bfloat16", 8, 4_096, 1_024, 1_024, "none", True, 2_048),
        # one new token for sixteen small networks
        rotary("rotary_token", "forward", "float32", 16, 1, 1, 4, 4, 64, 64, "half", "none", 200, 0),
        # eight small vision networks as above
        rotary("rotary_train", "train", "bfloat16", 8, 8, 197, 6, 6, 64, 32, "interleaved", "none", 0, 384),
        # long sequences beyond the trained context, shared key heads
        rotary("rotary_large_train", "train", "bfloat16", 8, 2, 4_096, 16, 4, 128, 128, "half", "parts", 1_000_000, 0),
        # one new token for sixteen small networks, 200 before it
        attention("attention_token", "forward", "float32", 16, 1, 1, 200, 4, 4, 64, causal=True),
        # one new token each for four long conversations with eight networks: reading the cache
        attention("attention_cache", "forward", "bfloat16", 8, 4, 1, 8_192, 16, 4, 128, causal=True, ragged=True),
        # eight small vision networks as above, every patch sees every other
        attention("attention_train", "train", "bfloat16", 8, 8, 197, 197, 6, 6, 64),
        # odd sizes, a learned slope for each head, single precision
        attention("attention_odd_train", "train", "float32", 3, 2, 333, 333, 6, 2, 40, causal=True, bias=True),
        # documents packed into sequences behind a common prefix, capped scores, half precision
        attention("attention_packed_train", "train", "float16", 4, 2, 2_000, 2_000, 8, 2, 64, causal=True, cap=30.0, prefix=64, documents=7),
        # long sequences of larger networks in mixed precision
        attention("attention_large_train", "train", "bfloat16", 4, 2, 4_096, 4_096, 16, 16, 64, causal=True),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e14)


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["linear", "rotary", "attention", "attention"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        c = {"op": op, "pass": rng.choice(["forward", "train"]), "type": rng.choice(list(_TYPES)), "n": _log_between(rng, 1, 32),
             "offset": rng.choice([0, 32 * rng.randint(1, 100), rng.randint(1, 10_000)])}
        if op == "linear":
            c |= {"rows": _log_between(rng, 1, 16_384), "width": _log_between(rng, 8, 2_048), "out": _log_between(rng, 8, 2_048)}
            if rng.random() < 0.5:
                c["width"], c["out"] = max(32, c["width"] // 32 * 32), max(32, c["out"] // 32 * 32)
            c |= {"act": rng.choice(["none", "none", "silu", "gelu", "relu", "tanh"]), "residual": rng.random() < 0.5}
        else:
            kv = _log_between(rng, 1, 8)
            c |= {"batch": _log_between(rng, 1, 8), "kv_heads": kv, "heads": kv * rng.choice([1, 1, 2, 3, 4]),
                  "dim": rng.choice([32, 64, 64, 128, rng.randint(4, 64) * 2])}
        if op == "rotary":
            c |= {"length": _log_between(rng, 1, 8_192), "norm": rng.random() < 0.8, "layout": rng.choice(["half", "interleaved"]),
                  "rotary": rng.choice([c["dim"], c["dim"], 2 * rng.randint(1, c["dim"] // 2)]), "scaling": rng.choice(["none", "linear", "parts"]),
                  "start": rng.choice([0, 0, _log_between(rng, 1, 2_000_000)]), "fused": rng.random() < 0.5}
        if op == "attention":
            c |= {"length": _log_between(rng, 1, 6_000), "causal": rng.random() < 0.7, "cap": rng.choice([0.0, 0.0, 20.0, 50.0]),
                  "bias": rng.random() < 0.3, "prefix": 0, "documents": 0, "ragged": False}
            c["keys"] = c["length"]
            kind = rng.choice(["same", "same", "cache", "prefix", "documents"])
            if kind == "cache":
                c |= {"length": rng.choice([1, 1, rng.randint(2, 40)]), "causal": True, "ragged": rng.random() < 0.5}
                c["keys"] = c["length"] + _log_between(rng, 1, 16_384)
            elif kind == "prefix":
                c |= {"causal": True, "prefix": rng.randint(1, c["length"])}
            elif kind == "documents":
                c["documents"] = rng.randint(1, 12)
        if _cost(c) <= most:
            return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _shapes(case):
    """The operator's parameters, in the order in which they lie in a row of X."""
    if case["op"] == "linear":
        return {"weight": (case["out"], case["width"]), "bias": (case["out"],)}
    if case["op"] == "rotary":
        return {"q_weight": (case["dim"],), "k_weight": (case["dim"],)} if case["norm"] else {}
    return {"slopes": (case["heads"],)} if case["bias"] else {}


def _views(matrix, case):
    views, at = {}, case["offset"]
    for name, shape in _shapes(case).items():
        size = math.prod(shape)
        views[name] = matrix[:, at:at + size].view(case["n"], *shape)
        at += size
    return views


def _rows_matrix(case):
    """An (n, D) view whose rows start on 128-byte boundaries, as the update likes them best."""
    D = case["offset"] + sum(math.prod(s) for s in _shapes(case).values())
    return torch.zeros(case["n"], (D + 32) // 32 * 32, device="cuda")[:, :D]


def _key_lengths(case):
    """How many keys of each sequence are filled: of a cache that ends at different places, the same for every seed."""
    rng = random.Random(case["keys"])
    return [case["keys"]] + [rng.randint(max(case["length"], case["keys"] // 2), case["keys"]) for _ in range(case["batch"] - 1)]


def _document_lengths(case):
    """Where each sequence's documents end: whole numbers that add up to its length, some of them 0."""
    rng = random.Random(case["keys"] + case["documents"])
    out = []
    for _ in range(case["batch"]):
        ends = sorted(rng.randint(0, case["keys"]) for _ in range(case["documents"] - 1)) + [case["keys"]]
        out.append([b - a for a, b in zip([0] + ends, ends)])
    return out


def _frequencies(case):
    """Angle per token of each rotated pair, in 64 bits."""
    r = case["rotary"]
    f = [BASE ** (-2.0 * j / r) for j in range(r // 2)]
    if case["scaling"] == "linear":
        f = [x / FACTOR for x in f]
    elif case["scaling"] == "parts":  # by how often a pair turns within the trained context: 32 times and more as it is, once and less stretched
        low, high = 1.0, 32.0
        for j, x in enumerate(f):
            keep = min(1.0, max(0.0, (TRAINED * x / (2.0 * math.pi) - low) / (high - low)))
            f[j] = x * (keep + (1.0 - keep) / FACTOR)
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, kind, train = case["n"], _TYPES[case["type"]], case["pass"] == "train"

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(kind)

    X, G = _rows_matrix(case), _rows_matrix(case)
    state = {"case": case, "X": X, "G": G, "params": _views(X, case), "grads": _views(G, case)}
    for name, p in state["params"].items():
        if name == "weight":
            p.copy_(torch.randn(p.shape, device="cuda", generator=gen) * case["width"] ** -0.5)
        elif name == "bias":
            p.copy_(torch.randn(p.shape, device="cuda", generator=gen) * 0.1)
        elif name == "slopes":  # a geometric row of them, each network's own by now
            h = torch.arange(1, case["heads"] + 1, device="cuda")
            p.copy_(torch.exp2(-8.0 * h / case["heads"]) * (1.0 + 0.1 * torch.randn(p.shape, device="cuda", generator=gen)))
        else:
            p.copy_(1.0 + 0.1 * torch.randn(p.shape, device="cuda", generator=gen))
    if case["op"] == "linear":
        rows = case["rows"]
        state["x"] = normal(n, rows, case["width"])
        if case["residual"]:
            state["residual"] = normal(n, rows, case["out"])
        if train:
            state["dy"] = normal(n, rows, case["out"], scale=1e-2)
        return state
    b, t, h, kv, d = case["batch"], case["length"], case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotary":
        if case["fused"]:
            qkv = normal(n, b, t, h + 2 * kv, d, scale=1.5)
            state["q"], state["k"] = qkv[..., :h, :], qkv[..., h:h + kv, :]
        else:
            state["q"], state["k"] = normal(n, b, t, h, d), normal(n, b, t, kv, d)
        if case["rotary"]:
            state["frequencies"] = _frequencies(case)
            state["positions"] = torch.arange(case["start"], case["start"] + t, device="cuda")
        if train:
            state["dq"], state["dk"] = normal(n, b, t, h, d, scale=1e-2), normal(n, b, t, kv, d, scale=1e-2)
        return state
    s = case["keys"]
    state["q"], state["k"], state["v"] = normal(n, b, t, h, d), normal(n, b, s, kv, d), normal(n, b, s, kv, d)
    masks = state["masks"] = {}
    if case["ragged"]:
        masks["lengths"] = torch.tensor(_key_lengths(case), dtype=torch.int32, device="cuda")
        masks["starts"] = masks["lengths"] - t
    if case["documents"]:
        masks["documents"] = torch.tensor([[i for i, m in enumerate(row) for _ in range(m)] for row in _document_lengths(case)],
                                          dtype=torch.int32, device="cuda")
    if case["prefix"]:
        masks["prefix"] = torch.full((b,), case["prefix"], dtype=torch.int32, device="cuda")
    if train:
        state["do"] = normal(n, b, t, h, d, scale=1e-2)
    return state


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _activation(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), (z > 0).float()
    if act == "tanh":
        a = torch.tanh(z)
        return a, 1.0 - a * a
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    cdf = 0.5 * torch.special.erfc(z * -(0.5 ** 0.5))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5


def _linear_plain(state, train):
    case, x, kind = state["case"], state["x"].float(), _TYPES[state["case"]["type"]]
    weight, bias = state["params"]["weight"], state["params"]["bias"]
    z = x @ weight.transpose(1, 2) + bias[:, None]
    a, slope = _activation(z, case["act"])
    y = a + state["residual"].float() if case["residual"] else a
    out = {"y": y.to(kind)}
    if train:
        dz = state["dy"].float() * slope
        out |= {"dx": (dz @ weight).to(kind), "dweight": dz.transpose(1, 2) @ x, "dbias": dz.sum(1)}
    return out


def _turn(x, cos, sin, layout):
    """The first 2 * cos.shape[-1] values of every head rotated; with -sin, rotated back."""
    r = 2 * cos.shape[-1]
    if r == 0:
        return x
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    c, s = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([c, s], -1) if layout == "half" else torch.stack([c, s], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _rotary_plain(state, train):
    case, kind = state["case"], _TYPES[state["case"]["type"]]
    if case["rotary"]:
        angle = state["positions"].double()[:, None] * state["frequencies"]
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    else:
        cos = sin = state["q"].new_zeros(0).float()
    out = {}
    for name in ("q", "k"):
        x = state[name].float()
        if case["norm"]:
            weight = state["params"][name + "_weight"][:, None, None, None]
            rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            xhat = x * rstd
            y = xhat * weight
        else:
            y = x
        out[name] = _turn(y, cos, sin, case["layout"]).to(kind)
        if train:
            g = _turn(state["d" + name].float(), cos, -sin, case["layout"])
            if case["norm"]:
                a = g * weight
                out["d" + name] = (rstd * (a - xhat * (a * xhat).mean(-1, keepdim=True))).to(kind)
                out[f"d{name}_weight"] = (g * xhat).sum((1, 2, 3))
            else:
                out["d" + name] = g.to(kind)
    return out


def _visible(state):
    """(batch, queries, keys): which keys a query sees, and the distances (queries, keys) or (batch, queries, keys)."""
    case, masks = state["case"], state["masks"]
    t, s = case["length"], case["keys"]
    j = torch.arange(s, device="cuda")
    p = torch.arange(t, device="cuda") + (masks["starts"][:, None] if "starts" in masks else s - t)
    p = p.reshape(-1, t, 1)
    see = torch.ones(1, t, s, dtype=torch.bool, device="cuda")
    if case["causal"]:
        see = j <= p
        if "prefix" in masks:
            see = see | (j < masks["prefix"][:, None, None])
    if "lengths" in masks:
        see = see & (j < masks["lengths"][:, None, None])
    if "documents" in masks:
        see = see & (masks["documents"][:, s - t:, None] == masks["documents"][:, None, :])
    return see, (p - j).abs().float()


def _attention_plain(state, train):
    case, kind = state["case"], _TYPES[state["case"]["type"]]
    n, b, t, s, h, kv, d = (case[k] for k in ("n", "batch", "length", "keys", "heads", "kv_heads", "dim"))
    group = h // kv
    see, distance = (m[:, None, None] for m in _visible(state))  # (batch or 1, 1, 1, queries, keys)
    at_a_time = max(1, 2 ** 30 // (b * h * t * s))
    parts = []
    for i in range(0, n, at_a_time):
        def heads(x, per):  # (particles, batch, kv heads, group, tokens, dim)
            x = x[i:i + at_a_time].float()
            return x.reshape(*x.shape[:3], kv, per, d).permute(0, 1, 3, 4, 2, 5).contiguous()
        q, k, v = heads(state["q"], group), heads(state["k"], 1), heads(state["v"], 1)
        score = (q @ k.transpose(-1, -2)) * d ** -0.5
        tanh = None
        if case["cap"]:
            tanh = torch.tanh(score / case["cap"])
            score = tanh * case["cap"]
        if case["bias"]:
            score = score - state["params"]["slopes"][i:i + at_a_time].reshape(-1, 1, kv, group, 1, 1) * distance
        score = score.masked_fill(~see, -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
        total = e.sum(-1, keepdim=True)
        p = e / torch.where(total == 0.0, 1.0, total)
        del score, e
        o = p @ v

        def back(x):  # (particles, batch, tokens, heads, dim)
            return x.permute(0, 1, 4, 2, 3, 5).flatten(3, 4).to(kind)
        part = {"o": back(o)}
        if train:
            do = heads(state["do"], group)
            ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True))
            part["dv"] = back((p.transpose(-1, -2) @ do).sum(3, keepdim=True))
            del p
            if case["bias"]:
                part["dslopes"] = -(ds * distance).sum((1, 4, 5)).reshape(-1, h)
            if tanh is not None:
                ds = ds * (1.0 - tanh * tanh)
            ds = ds * d ** -0.5
            part["dq"] = back(ds @ k)
            part["dk"] = back((ds.transpose(-1, -2) @ q).sum(3, keepdim=True))
        parts.append(part)
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]}


def run(state):
    case, train = state["case"], state["case"]["pass"] == "train"
    op, params, grads = case["op"], state["params"], state["grads"]
    if not own:
        return {"linear": _linear_plain, "rotary": _rotary_plain, "attention": _attention_plain}[op](state, train)
    from paper_2306_06528_amd import attention
    if op == "linear":
        y, saved = attention.linear_forward(state["x"], params["weight"], params["bias"], case["act"], state.get("residual"), save=train)
        if not train:
            return {"y": y}
        dx = attention.linear_backward(state["dy"], state["x"], params["weight"], saved, grads["weight"], grads["bias"], case["act"])
        return {"y": y, "dx": dx, "dweight": grads["weight"], "dbias": grads["bias"]}
    if op == "rotary":
        how = {"frequencies": state.get("frequencies"), "positions": state.get("positions"), "layout": case["layout"], "eps": EPS}
        weights = params.get("q_weight"), params.get("k_weight")
        q, k = attention.qk_norm_rotary_forward(state["q"], state["k"], *weights, **how)
        if not train:
            return {"q": q, "k": k}
        dweights = grads.get("q_weight"), grads.get("k_weight")
        dq, dk = attention.qk_norm_rotary_backward(state["dq"], state["dk"], state["q"], state["k"], *weights, *dweights, **how)
        out = {"q": q, "k": k, "dq": dq, "dk": dk}
        return out | {"dq_weight": dweights[0], "dk_weight": dweights[1]} if case["norm"] else out
    how = {"causal": case["causal"], "cap": case["cap"], "slopes": params.get("slopes"), **state["masks"]}
    o, lse = attention.attention_forward(state["q"], state["k"], state["v"], **how)
    if not train:
        return {"o": o}
    dq, dk, dv = attention.attention_backward(state["do"], state["q"], state["k"], state["v"], o, lse, dslopes=grads.get("slopes"), **how)
    out = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    return out | {"dslopes": grads["slopes"]} if case["bias"] else out


def _pairs(case):
    """Queries and the keys they see, over the batch."""
    t, s, b, prefix = case["length"], case["keys"], case["batch"], case["prefix"]

    def seen(first, last, low, high):  # queries at positions first .. last - 1, keys low .. high - 1
        if not case["causal"]:
            return (last - first) * (high - low)
        return sum(max(0, min(high, max(i + 1, prefix)) - low) for i in range(first, last))
    if case["ragged"]:
        return sum(seen(m - t, m, 0, m) for m in _key_lengths(case))
    if not case["documents"]:
        return b * seen(s - t, s, 0, s)
    total = 0
    for row in _document_lengths(case):
        at = 0
        for m in row:
            total += seen(max(at, s - t), at + m, at, at + m) if at + m > s - t else 0
            at += m
    return total


def work(case):
    n, train = case["n"], case["pass"] == "train"
    size = {"float32": 4, "bfloat16": 2, "float16": 2}[case["type"]]
    params = 4 * n * sum(math.prod(s) for s in _shapes(case).values()) * (2 if train else 1)
    if case["op"] == "linear":
        rows, d, f = case["rows"], case["width"], case["out"]
        acts = rows * (d + f) * (2 if train else 1) + (rows * f if case["residual"] else 0)
        return {"bytes": size * n * acts + params, "flops": 2 * n * rows * d * f * (3 if train else 1)}
    b, t, h, kv, d = case["batch"], case["length"], case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotary":
        values = n * b * t * (h + kv) * d
        return {"bytes": size * values * (4 if train else 2) + params, "flops": values * (22 if train else 8)}
    keys = sum(_key_lengths(case)) if case["ragged"] else b * case["keys"]
    acts = n * d * (b * t * h * 2 + keys * kv * 2)  # q and o, k and v; do and dq, dk and dv
    return {"bytes": size * acts * (2 if train else 1) + params, "flops": (14 if train else 4) * n * h * d * _pairs(case)}


# ---------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_linear(state, i):
    case, x = state["case"], state["x"][i].double()
    weight, bias = (state["params"][k][i].double() for k in ("weight", "bias"))
    z = torch.addmm(bias, x, weight.t())
    if case["act"] == "silu":
        s = torch.sigmoid(z)
        a, slope = z * s, s + z * s * (1 - s)
    elif case["act"] == "gelu":
        s = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        a, slope = z * s, s + z * torch.exp(-z.square() / 2) / math.sqrt(2.0 * math.pi)
    elif case["act"] == "tanh":
        a, slope = torch.tanh(z), torch.cosh(z).pow(-2)
    elif case["act"] == "relu":
        a, slope = z.clamp(min=0), torch.sign(z).clamp(min=0)
    else:
        a, slope = z, torch.ones_like(z)
    out = {"y": a + state["residual"][i].double() if case["residual"] else a}
    if "dy" in state:
        dz = state["dy"][i].double() * slope
        out |= {"dx": torch.mm(dz, weight), "dweight": torch.mm(dz.t(), x), "dbias": dz.sum(0)}
    return out


def _exact_rotary(state, i):
    """The pairs as complex numbers, turned by exp(i angle)."""
    case, out, r = state["case"], {}, state["case"]["rotary"]

    def turned(x, back):
        if not r:
            return x
        w = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), torch.outer(state["positions"].double(), state["frequencies"]))[:, None]
        w = w.conj() if back else w
        head, rest = x[..., :r], x[..., r:]
        pairs = head.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else head.unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * w)
        return torch.cat([(z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2), rest], -1)
    for name in ("q", "k"):
        x = state[name][i].double()
        sigma = torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + EPS) if case["norm"] else torch.ones_like(x[..., :1])
        weight = state["params"][name + "_weight"][i].double() if case["norm"] else torch.ones_like(x[0, 0, 0])
        out[name] = turned(x / sigma * weight, False)
        if "dq" in state:
            g = turned(state["d" + name][i].double(), True)
            dxhat = g * weight
            dx = dxhat / sigma
            if case["norm"]:
                dx = dx - x * (dxhat * x).sum(-1, keepdim=True) / (case["dim"] * sigma ** 3)
                out[f"d{name}_weight"] = torch.einsum("bthd,bthd->d", g, x / sigma)
            out["d" + name] = dx
    return out


def _exact_attention(state, i):
    case, masks = state["case"], state["masks"]
    t, s, h, kv, d = (case[k] for k in ("length", "keys", "heads", "kv_heads", "dim"))
    rows, columns = torch.arange(t, device="cuda")[:, None], torch.arange(s, device="cuda")[None]
    out = {name: torch.zeros_like(state[like][i], dtype=torch.float64) for name, like in
           (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    out["dslopes"] = torch.zeros(h, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        first = int(masks["starts"][b]) if "starts" in masks else s - t
        hidden = torch.zeros(t, s, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = (columns > rows + first) & (columns >= case["prefix"])
        if "lengths" in masks:
            hidden = hidden | (columns >= int(masks["lengths"][b]))
        if "documents" in masks:
            hidden = hidden | (masks["documents"][b, s - t:, None] != masks["documents"][b])
        far = (rows + first - columns).abs().double()
        for head in range(h):
            q, k, v = state["q"][i, b, :, head].double(), state["k"][i, b, :, head // (h // kv)].double(), state["v"][i, b, :, head // (h // kv)].double()
            z = torch.mm(q, k.t()) / math.sqrt(d)
            slope = 1.0
            if case["cap"]:
                slope = torch.cosh(z / case["cap"]).pow(-2)
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["bias"]:
                z = z - state["params"]["slopes"][i, head].double() * far
            z = z.masked_fill(hidden, -math.inf)
            p = torch.exp(z - torch.logsumexp(z, -1, keepdim=True)).nan_to_num(nan=0.0)  # (rows that see nothing)
            o = torch.mm(p, v)
            out["o"][b, :, head] = o
            if "do" not in state:
                continue
            do = state["do"][i, b, :, head].double()
            dz = p * (torch.mm(do, v.t()) - (do * o).sum(-1, keepdim=True))
            out["dslopes"][head] -= (dz * far).sum()
            dz = dz * slope / math.sqrt(d)
            out["dq"][b, :, head] = torch.mm(dz, k)
            out["dk"][b, :, head // (h // kv)] += torch.mm(dz.t(), q)
            out["dv"][b, :, head // (h // kv)] += torch.mm(p.t(), do)
    keep = {"o"} | ({"dq", "dk", "dv"} | ({"dslopes"} if case["bias"] else set()) if "do" in state else set())
    return {k: v for k, v in out.items() if k in keep}


def exact(case, seed):
    state = prepare(case, seed)
    one = {"linear": _exact_linear, "rotary": _exact_rotary, "attention": _exact_attention}[case["op"]]
    each = [one(state, i) for i in range(case["n"])]
    return {k: torch.stack([e[k] for e in each]) for k in each[0]}
