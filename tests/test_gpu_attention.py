"""The attention half of the particles' layers on the GPU against the definitions in 64 bits (tests/attention_reference.py: every value within the bound that
roundings allow), over types, sizes around the kernels' tiles, head layouts, masks, strides and special values."""
import math
import zlib

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def gen(*key):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def params(g, n, at, *shapes, spread=1.0):
    """Parameters and (poisoned) gradients, side by side in the rows of X and G from column `at` on."""
    D = at + sum(math.prod(s) for s in shapes) + 3
    X, G = torch.full((n, D), float("nan"), device="cuda"), torch.full((n, D), -7.0, device="cuda")
    views, grads = [], []
    for s in shapes:
        size = math.prod(s)
        v = X[:, at:at + size].view(n, *s)
        v.copy_((torch.randn(n, *s, generator=g) * spread).cuda())
        views.append(v)
        grads.append(G[:, at:at + size].view(n, *s))
        at += size
    return views, grads, G, D


def untouched(G, first, last):
    assert (G[:, :first] == -7.0).all() and (G[:, last:] == -7.0).all()


def normal(g, *shape, dtype, scale=1.0, layout="dense"):
    v = (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()
    if layout == "dense":
        return v
    if layout == "gap":  # rows off the 16-byte boundaries, something between them
        buf = torch.full((*shape[:-2], shape[-2] + 1, shape[-1] + 5), float("nan"), dtype=dtype, device="cuda")
        return buf[..., :shape[-2], 3:3 + shape[-1]].copy_(v)
    if layout == "transposed":  # heads (or rows) before what comes before them
        return v.transpose(-2, -3).contiguous().transpose(-2, -3)
    assert layout == "shared"
    return v[:1].expand(shape[0], *[-1] * (len(shape) - 1))


# ---------------------------------------------------------------------------------------------
# linear map
# ---------------------------------------------------------------------------------------------
LINEAR_SIZES = [(1, 1, 1, 1), (2, 3, 5, 2), (3, 5, 33, 17), (2, 16, 64, 48), (1, 17, 100, 31), (2, 32, 96, 130), (2, 33, 40, 65), (1, 70, 129, 257), (2, 200, 64, 96), (1, 300, 515, 260),
                (64, 2, 8, 8), (1, 1, 3000, 5), (1, 130, 2000, 40), (2, 5, 7, 1025), (1, 700, 3, 2)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,out", LINEAR_SIZES)
def test_linear(att, n, rows, width, out, dtype):
    g = gen(n, rows, width, out)
    act = ["none", "silu", "gelu", "relu", "tanh"][(rows + width) % 5]
    x, dy = normal(g, n, rows, width, dtype=dtype), normal(g, n, rows, out, dtype=dtype)
    residual = normal(g, n, rows, out, dtype=dtype) if out % 2 else None
    (w, b), (dw, db), G, D = params(g, n, 5, (out, width), (out,))
    for a in {act, "none"}:
        G.fill_(-7.0)
        y, saved = att.linear_forward(x, w, b, a, residual, save=True)
        dx = att.linear_backward(dy, x, w, saved, dw, db, a)
        want = ref.linear(x, w, b, a, residual, dy)
        for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
            ref.check(got, want[name], f"{name} of {n}x{rows}x{width}x{out} {a}")
        untouched(G, 5, D - 3)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu", "tanh"])
@pytest.mark.parametrize("layout", ["gap", "transposed", "shared"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,out", [(3, 10, 24, 40), (2, 150, 130, 70)])
def test_linear_layouts(att, n, rows, width, out, dtype, layout, act):
    g = gen(n, rows, act)
    x, dy, residual = (normal(g, n, rows, m, dtype=dtype, layout=layout) for m in (width, out, out))
    (w, b), (dw, db), G, D = params(g, n, 2, (out, width), (out,))
    y, saved = att.linear_forward(x, w, b, act, residual, save=True)
    dx = att.linear_backward(dy, x, w, saved, dw, db, act)
    want = ref.linear(x, w, b, act, residual, dy)
    for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
        ref.check(got, want[name], name)
    assert torch.equal(att.linear_forward(x, w, b, act, residual)[0], y)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("n,rows,width,out", [(8, 1_576, 384, 1_153), (4, 2_050, 1_030, 1_029), (20, 333, 500, 500), (2, 3_001, 97, 600)])
def test_linear_large(att, n, rows, width, out, act, dtype):
    """Tiles of every kind, with the columns whole and in parts."""
    g = gen(rows, act)
    x, dy = normal(g, n, rows, width, dtype=dtype), normal(g, n, rows, out, dtype=dtype)
    (w, b), (dw, db), G, D = params(g, n, 3, (out, width), (out,), spread=width ** -0.5)
    y, saved = att.linear_forward(x, w, b, act, save=True)
    dx = att.linear_backward(dy, x, w, saved, dw, db, act)
    want = ref.linear(x, w, b, act, None, dy)
    for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
        ref.check(got, want[name], name)
    untouched(G, 3, D - 3)


def test_linear_parts_and_accumulate(att):
    g = gen(1)
    for rows in (9, 100):
        x, dy = normal(g, 2, rows, 50, dtype=torch.float32), normal(g, 2, rows, 20, dtype=torch.float32)
        (w, b), (dw, db), G, D = params(g, 2, 0, (20, 50), (20,))
        y, saved = att.linear_forward(x, w)  # no bias
        assert saved is None
        ref.check(y, ref.linear(x, w, None, "none")["y"], "y without a bias")
        dx = att.linear_backward(dy, x, w, None, dw, db)
        first = G.clone()
        assert torch.equal(att.linear_backward(dy, x, w), dx) and torch.equal(G, first)
        assert att.linear_backward(dy, x, w, None, None, db, want_dx=False) is None and torch.equal(G, first)
        att.linear_backward(dy, x, w, None, dw, db, accumulate=True)
        assert torch.equal(dw, 2 * first[:, :1000].view(2, 20, 50)) and torch.equal(db, 2 * first[:, 1000:1020])


def test_linear_no_rows(att):
    g = gen(2)
    (w, b), (dw, db), G, D = params(g, 2, 0, (6, 4), (6,))
    x, dy = torch.zeros(2, 0, 4, device="cuda"), torch.zeros(2, 0, 6, device="cuda")
    for act in ("none", "gelu"):
        G.fill_(-7.0)
        y, saved = att.linear_forward(x, w, b, act, save=True)
        assert y.shape == (2, 0, 6)
        att.linear_backward(dy, x, w, saved, dw, db, act, accumulate=True)
        assert (G == -7.0).all()
        att.linear_backward(dy, x, w, saved, dw, db, act)
        assert (dw == 0).all() and (db == 0).all()
        untouched(G, 0, D - 3)


def test_linear_more_dimensions(att):
    g = gen(3)
    x = normal(g, 2, 3, 5, 8, dtype=torch.bfloat16)
    (w, b), (dw, db), _, _ = params(g, 2, 0, (6, 8), (6,))
    y, saved = att.linear_forward(x, w, b, "silu", save=True)
    assert y.shape == (2, 3, 5, 6)
    ref.check(y.flatten(1, 2), ref.linear(x.flatten(1, 2), w, b, "silu")["y"], "y")
    dy = normal(g, 2, 3, 5, 6, dtype=torch.bfloat16)
    assert att.linear_backward(dy, x, w, saved, dw, db, "silu").shape == x.shape


# ---------------------------------------------------------------------------------------------
# norms and rotation
# ---------------------------------------------------------------------------------------------
ROTARY = [  # n, batch, tokens, heads, kv_heads, dim, pairs, layout, start
    (2, 1, 1, 1, 1, 2, 1, "half", 0), (1, 2, 3, 2, 1, 7, 3, "interleaved", 5), (3, 2, 5, 4, 2, 64, 32, "half", 1_000_000), (2, 1, 9, 3, 3, 40, 20, "half", 7),
    (2, 3, 17, 2, 1, 128, 64, "interleaved", 0), (1, 1, 40, 5, 1, 96, 17, "half", 30), (2, 2, 6, 2, 2, 256, 128, "half", 0), (1, 2, 11, 3, 1, 255, 100, "interleaved", 12),
    (2, 1, 700, 2, 1, 32, 16, "half", 0), (64, 1, 2, 1, 1, 8, 4, "half", 3), (2, 2, 4, 2, 1, 64, 0, "half", 0), (1, 1, 3, 1, 2, 130, 65, "half", 2_000_000)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("layout_in", ["fused", "gap", "transposed", "shared"])
@pytest.mark.parametrize("n,batch,t,heads,kv,dim,pairs,layout,start", ROTARY)
def test_rotary(att, n, batch, t, heads, kv, dim, pairs, layout, start, layout_in, norm, dtype):
    g = gen(n, t, dim, pairs)
    if layout_in == "fused":
        both = normal(g, n, batch, t, heads + 2 * kv, dim, dtype=dtype, scale=1.5)
        q, k = both[..., :heads, :], both[..., heads:heads + kv, :]
        dboth = normal(g, n, batch, t, heads + 2 * kv, dim, dtype=dtype)
        dq, dk = dboth[..., :heads, :], dboth[..., heads:heads + kv, :]
    else:
        q, dq = (normal(g, n, batch, t, heads, dim, dtype=dtype, layout=layout_in) for _ in range(2))
        k, dk = (normal(g, n, batch, t, kv, dim, dtype=dtype, layout=layout_in) for _ in range(2))
    (qw, kw), (dqw, dkw), G, D = params(g, n, 3, (dim,), (dim,))
    frequencies = torch.tensor([10_000.0 ** (-2 * j / dim) for j in range(pairs)], dtype=torch.float64, device="cuda") if pairs else None
    positions = torch.arange(start, start + t, device="cuda") if pairs else None
    if pairs and batch > 1:  # every sequence its own
        positions = (positions[None] + 3 * torch.arange(batch, device="cuda")[:, None]).contiguous()
    weights = (qw, kw) if norm else (None, None)
    how = {"frequencies": frequencies, "positions": positions, "layout": layout, "eps": 1e-6}
    got = dict(zip(("q", "k"), att.qk_norm_rotary_forward(q, k, *weights, **how)))
    got |= dict(zip(("dq", "dk"), att.qk_norm_rotary_backward(dq, dk, q, k, *weights, *((dqw, dkw) if norm else (None, None)), **how)))
    for name, x, w, dy, dw in (("q", q, weights[0], dq, dqw), ("k", k, weights[1], dk, dkw)):
        want = ref.qk_norm_rotary(x, w, frequencies, positions, layout, 1e-6, dy)
        ref.check(got[name], want["y"], name)
        ref.check(got["d" + name], want["dx"], "d" + name)
        if norm:
            ref.check(dw, want["dweight"], f"d{name}_weight")
    untouched(G, 3, D - 3 if norm else 3)


def test_rotary_parts_and_accumulate(att):
    g = gen(5)
    q, k, dq, dk = (normal(g, 2, 2, 9, h, 24, dtype=torch.float32) for h in (4, 2, 4, 2))
    (qw, kw), (dqw, dkw), G, D = params(g, 2, 0, (24,), (24,))
    args = (dq, dk, q, k, qw, kw)
    first = att.qk_norm_rotary_backward(*args, dqw, dkw)
    once = G.clone()
    again = att.qk_norm_rotary_backward(*args)
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(G, once)
    att.qk_norm_rotary_backward(*args, None, dkw)
    assert torch.equal(G, once)
    att.qk_norm_rotary_backward(*args, dqw, None, accumulate=True)
    assert torch.equal(dqw, 2 * once[:, :24]) and torch.equal(dkw, once[:, 24:48])
    empty = [x[:, :, :0] for x in (dq, dk, q, k)]
    att.qk_norm_rotary_backward(*empty, qw, kw, dqw, dkw, accumulate=True)
    assert torch.equal(dqw, 2 * once[:, :24])
    att.qk_norm_rotary_backward(*empty, qw, kw, dqw, dkw)
    assert (dqw == 0).all() and (dkw == 0).all()


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------
def run_attention(att, q, k, v, do, **how):
    """Forward and backward against the definitions."""
    n, heads = q.shape[0], q.shape[3]
    slopes, ds = how.get("slopes"), None
    if slopes is not None:
        G = torch.full((n, heads + 4), -7.0, device="cuda")
        ds = G[:, 2:2 + heads]
    o, lse = att.attention_forward(q, k, v, **how)
    got = {"o": o}
    got |= dict(zip(("dq", "dk", "dv"), att.attention_backward(do, q, k, v, o, lse, dslopes=ds, **how)))
    if slopes is not None:
        got["dslopes"] = ds
        assert (G[:, :2] == -7.0).all() and (G[:, 2 + heads:] == -7.0).all()
    want = ref.attention(q, k, v, do, **how)
    for name, x in got.items():
        ref.check(x, want[name], name)
    ref.check_lse(lse, want["lse"])
    return got, lse


SIZES = [  # n, batch, tokens, keys, heads, kv_heads, dim
    (1, 1, 1, 1, 1, 1, 1), (2, 1, 2, 3, 2, 1, 8), (1, 2, 15, 17, 3, 3, 33), (2, 1, 64, 64, 2, 2, 32), (1, 2, 65, 65, 4, 2, 64), (1, 1, 130, 129, 2, 1, 40), (2, 2, 33, 200, 4, 1, 80),
    (1, 1, 197, 197, 3, 3, 64), (1, 1, 70, 300, 6, 2, 96), (1, 1, 129, 257, 2, 2, 127), (1, 1, 260, 140, 4, 2, 128), (3, 1, 1, 500, 4, 4, 64), (1, 3, 1, 1_000, 8, 2, 128), (2, 1, 5, 700, 6, 2, 50),
    (64, 1, 2, 4, 1, 1, 16)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,batch,t,s,heads,kv,d", SIZES)
def test_attention(att, n, batch, t, s, heads, kv, d, causal, dtype):
    g = gen(n, t, s, d)
    q, do = normal(g, n, batch, t, heads, d, dtype=dtype), normal(g, n, batch, t, heads, d, dtype=dtype)
    k, v = normal(g, n, batch, s, kv, d, dtype=dtype), normal(g, n, batch, s, kv, d, dtype=dtype)
    run_attention(att, q, k, v, do, causal=causal)  # (more queries than keys: the first ones see nothing)


def masks_of(kind, g, batch, t, s):
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    if kind == "lengths":  # none, one, odd ones, all, more than there are
        return {"lengths": ints([[0, 1, s // 2 + 1, s, s + 9][(b + 2) % 5] for b in range(batch)])}
    if kind == "ragged":
        lengths = ints([max(t, s - 7 * b) for b in range(batch)])
        return {"causal": True, "lengths": lengths, "starts": lengths - t}
    if kind == "starts":  # before the first key, behind the last one
        return {"causal": True, "starts": ints([[-3, s - 1, 2, s + 5, -2 * t][b % 5] for b in range(batch)])}
    if kind == "prefix":
        return {"causal": True, "prefix": ints([[0, s // 3, s, 1, s + 4][(b + 1) % 5] for b in range(batch)])}
    if kind == "documents":
        return {"documents": ints([sorted(torch.randint(0, 5, (s,), generator=g).tolist()) for _ in range(batch)])}
    if kind == "mixed_documents":  # in no order, some of them negative
        return {"causal": True, "documents": torch.randint(-2, 3, (batch, s), generator=g, dtype=torch.int32).cuda()}
    assert kind == "everything"
    return {"causal": True, "documents": ints([sorted(torch.randint(0, 4, (s,), generator=g).tolist()) for _ in range(batch)]), "prefix": ints([s // 4] * batch),
            "lengths": ints([s - 3 * b for b in range(batch)]), "starts": ints([s - t - b for b in range(batch)])}


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["lengths", "ragged", "starts", "prefix", "documents", "mixed_documents", "everything"])
@pytest.mark.parametrize("t,s,heads,kv,d", [(30, 45, 4, 2, 24), (150, 150, 2, 1, 64), (70, 333, 3, 3, 100), (1, 600, 4, 1, 64)])
def test_attention_masks(att, t, s, heads, kv, d, kind, dtype):
    batch = 5
    g = gen(t, s, kind)
    q, do = normal(g, 1, batch, t, heads, d, dtype=dtype), normal(g, 1, batch, t, heads, d, dtype=dtype)
    k, v = normal(g, 1, batch, s, kv, d, dtype=dtype), normal(g, 1, batch, s, kv, d, dtype=dtype)
    how = masks_of(kind, g, batch, t, s)
    if "lengths" in how:  # what lies behind is not read
        for b in range(batch):
            k[:, b, max(0, int(how["lengths"][b])):] = float("nan")
            v[:, b, max(0, int(how["lengths"][b])):] = float("inf")
    run_attention(att, q, k, v, do, **how)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("cap,bias", [(5.0, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("n,batch,t,s,heads,kv,d", [(2, 2, 40, 40, 4, 2, 32), (1, 2, 200, 200, 3, 1, 72), (2, 1, 3, 400, 2, 2, 128), (1, 1, 130, 90, 2, 1, 96)])
def test_attention_scores(att, n, batch, t, s, heads, kv, d, cap, bias, dtype):
    g = gen(n, t, s, cap)
    q, do = normal(g, n, batch, t, heads, d, dtype=dtype, scale=2.0), normal(g, n, batch, t, heads, d, dtype=dtype)
    k, v = normal(g, n, batch, s, kv, d, dtype=dtype, scale=2.0), normal(g, n, batch, s, kv, d, dtype=dtype)
    slopes = None
    if bias:
        (slopes,), _, _, _ = params(g, n, 1, (heads,), spread=0.1)
    for causal in (False, True):
        run_attention(att, q, k, v, do, causal=causal, cap=cap, slopes=slopes)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", ["gap", "transposed", "shared"])
def test_attention_layouts(att, layout, dtype):
    g = gen(layout)
    for n, batch, t, s, heads, kv, d in ((2, 2, 70, 70, 4, 2, 48), (2, 1, 5, 300, 3, 1, 63)):
        q, do = (normal(g, n, batch, t, heads, d, dtype=dtype, layout=layout) for _ in range(2))
        k, v = (normal(g, n, batch, s, kv, d, dtype=dtype, layout=layout) for _ in range(2))
        run_attention(att, q, k, v, do, causal=True, scale=0.2)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_attention_large_scores(att, dtype):
    """Scores far from zero, rising from tile to tile: the running maximum; gradients far from 1 (fp16's range)."""
    g = gen(9)
    t, s, d = 100, 400, 64
    q, k = normal(g, 1, 1, t, 2, d, dtype=dtype, scale=3.0), normal(g, 1, 1, s, 2, d, dtype=dtype, scale=3.0)
    k = (k.float() * torch.linspace(0.1, 2.0, s, device="cuda")[None, None, :, None, None]).to(dtype)
    v = normal(g, 1, 1, s, 2, d, dtype=dtype)
    for size in (1e-5, 1.0, 1e3):
        run_attention(att, q, k, v, normal(g, 1, 1, t, 2, d, dtype=dtype, scale=size))


def test_attention_nothing(att):
    """No queries, no keys, no sequences."""
    g = gen(10)
    for batch, t, s in ((2, 0, 5), (2, 3, 0), (0, 3, 4), (1, 0, 0)):
        q, do = normal(g, 2, batch, t, 4, 16, dtype=torch.bfloat16), normal(g, 2, batch, t, 4, 16, dtype=torch.bfloat16)
        k, v = normal(g, 2, batch, s, 2, 16, dtype=torch.bfloat16), normal(g, 2, batch, s, 2, 16, dtype=torch.bfloat16)
        (slopes,), (ds,), G, _ = params(g, 2, 0, (4,))
        o, lse = att.attention_forward(q, k, v, slopes=slopes)
        assert o.shape == q.shape and (o == 0).all() and (lse == -math.inf).all()
        before = ds.clone()
        dq, dk, dv = att.attention_backward(do, q, k, v, o, lse, slopes=slopes, dslopes=ds, accumulate=True)
        assert torch.equal(ds, before) and all((x == 0).all() for x in (dq, dk, dv)) and dk.shape == k.shape
        att.attention_backward(do, q, k, v, o, lse, slopes=slopes, dslopes=ds)
        assert (ds == 0).all()


def test_attention_parts(att):
    g = gen(11)
    q, do = (normal(g, 2, 2, 50, 4, 32, dtype=torch.bfloat16) for _ in range(2))
    k, v = (normal(g, 2, 2, 50, 2, 32, dtype=torch.bfloat16) for _ in range(2))
    (slopes,), (ds,), G, _ = params(g, 2, 0, (4,), spread=0.1)
    o, lse = att.attention_forward(q, k, v, causal=True, slopes=slopes)
    all_of = att.attention_backward(do, q, k, v, o, lse, causal=True, slopes=slopes, dslopes=ds)
    once = ds.clone()
    some = att.attention_backward(do, q, k, v, o, lse, causal=True, slopes=slopes, want_dq=False)
    assert some[0] is None and torch.equal(some[1], all_of[1]) and torch.equal(some[2], all_of[2])
    some = att.attention_backward(do, q, k, v, o, lse, causal=True, slopes=slopes, dslopes=ds, accumulate=True, want_dkv=False)
    assert some[1] is None and some[2] is None and torch.equal(some[0], all_of[0]) and torch.equal(ds, 2 * once)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["causal", "documents", "prefix"])
@pytest.mark.parametrize("n,batch,t,s,heads,kv,d", [(2, 5, 1_100, 1_100, 3, 3, 24), (1, 5, 540, 700, 4, 2, 40), (5, 7, 330, 330, 2, 1, 72), (3, 4, 200, 1_000, 3, 3, 100)])
def test_attention_uneven_workgroups(att, n, batch, t, s, heads, kv, d, kind, dtype):
    """Workgroups whose masks leave them unlike numbers of tiles: streamed rows in parts, up to 682 workgroups; heads that all take turns (up to 31 key heads) or four at a time."""
    g = gen(n, t, s, heads, kind)
    how = {"causal": True} if kind == "causal" else masks_of(kind, g, batch, t, s) | {"causal": True}
    q, do = (normal(g, n, batch, t, heads, d, dtype=dtype) for _ in range(2))
    k, v = (normal(g, n, batch, s, kv, d, dtype=dtype) for _ in range(2))
    run_attention(att, q, k, v, do, **how)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("how", [{"causal": True}, {"cap": 8.0}], ids=["causal", "cap"])
@pytest.mark.parametrize("n,batch,t,s,heads,kv,d", [(16, 16, 130, 130, 8, 8, 24), (24, 16, 135, 150, 12, 4, 64), (16, 20, 70, 200, 4, 4, 90), (16, 12, 140, 140, 8, 8, 120), (32, 64, 66, 66, 2, 2, 5)])
def test_attention_many_workgroups(att, n, batch, t, s, heads, kv, d, how, dtype):
    """So many that a wave has two blocks of rows or of keys: some sequences against the definitions."""
    g = torch.Generator(device="cuda").manual_seed(t + d)
    make = lambda tokens, h: torch.randn(n, batch, tokens, h, d, generator=g, device="cuda").to(dtype)  # noqa: E731
    q, do, k, v = make(t, heads), make(t, heads), make(s, kv), make(s, kv)
    o, lse = att.attention_forward(q, k, v, **how)
    got = (o, *att.attention_backward(do, q, k, v, o, lse, **how))
    for i, b in ((0, 0), (n - 1, batch - 1), (n // 2, 3)):
        part = lambda x: x[i:i + 1, b:b + 1]  # noqa: E731
        want = ref.attention(part(q), part(k), part(v), part(do), **how)
        for name, x in zip(("o", "dq", "dk", "dv"), got):
            ref.check(part(x), want[name], f"{name} of {i}, {b}")
        ref.check_lse(part(lse), want["lse"])
