"""The particles' layers on the GPU against their definitions in 64 bits (tests/layer_reference.py: every value within the bound
that roundings allow), over types, sizes around the kernels' tiles, strides, alignments and special values."""
import math

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def layers():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import layers as mod
    return mod


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def acts(g, n, rows, width, dtype, layout="dense", scale=1.0, shift=0.0):
    """Activations in one of the layouts that a caller may have."""
    v = (torch.randn(n, rows, width, generator=g) * scale + shift).to(dtype).cuda()
    if layout == "dense":
        return v
    if layout == "gap":  # rows off the 16-byte boundaries, something between them
        buf = torch.full((n, rows + 1, width + 5), float("nan"), dtype=dtype, device="cuda")
        out = buf[:, :rows, 3:3 + width]
        return out.copy_(v)
    if layout == "rows_first":
        return v.transpose(0, 1).contiguous().transpose(0, 1)
    assert layout == "shared"
    return v[:1].expand(n, -1, -1)


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
    """What lies before and behind the layer's gradients in the rows of G is as it was."""
    assert (G[:, :first] == -7.0).all() and (G[:, last:] == -7.0).all()


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------
NORM_SIZES = [(1, 1, 1), (2, 3, 2), (3, 5, 7), (2, 33, 8), (2, 40, 63), (2, 9, 65), (2, 17, 128), (1, 10, 129), (2, 70, 256), (3, 5, 257), (2, 6, 511),
              (2, 9, 513), (1, 11, 1023), (2, 3, 1025), (1, 4, 2048), (1, 3, 2049), (1, 2, 4097), (2, 3, 8191), (1, 2, 8193), (1, 2, 16384), (64, 2, 5)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width", NORM_SIZES)
def test_norm(layers, n, rows, width, dtype):
    g = gen(n, rows, width)
    x, dy = acts(g, n, rows, width, dtype, shift=0.5), acts(g, n, rows, width, dtype)
    (w, b), (dw, db), G, D = params(g, n, 5, (width,), (width,))
    eps = 1e-5
    y, mean, rstd = layers.layer_norm_forward(x, w, b, eps)
    dx = layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db)
    want = ref.layer_norm(x, w, b, eps, dy)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dweight", dw), ("dbias", db)):
        ref.check(got, want[name], f"{name} of {n}x{rows}x{width}")
    untouched(G, 5, D - 3)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", ["gap", "rows_first", "shared"])
@pytest.mark.parametrize("n,rows,width", [(3, 10, 24), (2, 7, 1001)])
def test_norm_layouts(layers, n, rows, width, layout, dtype):
    g = gen(n, rows, width, 1)
    x, dy = acts(g, n, rows, width, dtype, layout), acts(g, n, rows, width, dtype, layout)
    (w, b), (dw, db), G, D = params(g, n, 1, (width,), (width,))
    y, mean, rstd = layers.layer_norm_forward(x, w, b)
    dx = layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db)
    want = ref.layer_norm(x, w, b, 1e-5, dy)
    for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
        ref.check(got, want[name], name)


def test_norm_many_rows(layers):
    """Many workgroups per particle, ragged ends, the partial sums of all of them."""
    g = gen(2)
    for n, rows, width in ((3, 4_099, 40), (1, 20_011, 17), (7, 1_301, 300)):
        x, dy = acts(g, n, rows, width, torch.float32), acts(g, n, rows, width, torch.float32)
        (w, b), (dw, db), _, _ = params(g, n, 0, (width,), (width,))
        y, mean, rstd = layers.layer_norm_forward(x, w, b)
        dx = layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db)
        want = ref.layer_norm(x, w, b, 1e-5, dy)
        for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
            ref.check(got, want[name], name)


def test_norm_far_from_zero(layers):
    """The mean is taken off before squares are summed: rows at 1000 with a spread of 1 keep their digits."""
    g = gen(3)
    x = acts(g, 2, 5, 700, torch.float32, shift=1000.0)
    (w, b), _, _, _ = params(g, 2, 0, (700,), (700,))
    y, mean, rstd = layers.layer_norm_forward(x, w, b)
    want = ref.layer_norm(x, w, b, 1e-5)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd)):
        ref.check(got, want[name], name)


def test_norm_parts_and_accumulate(layers):
    g = gen(4)
    n, rows, width = 2, 9, 50
    x, dy = acts(g, n, rows, width, torch.float32), acts(g, n, rows, width, torch.float32)
    (w, b), (dw, db), G, D = params(g, n, 0, (width,), (width,))
    y0, mean, rstd = layers.layer_norm_forward(x, w)  # no bias
    ref.check(y0, ref.layer_norm(x, w, None, 1e-5)["y"], "y without a bias")
    dx = layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db)
    first = G.clone()
    assert torch.equal(layers.layer_norm_backward(dy, x, w, mean, rstd), dx)
    assert torch.equal(G, first)
    assert layers.layer_norm_backward(dy, x, w, mean, rstd, None, db, want_dx=False) is None
    assert torch.equal(G, first)
    layers.layer_norm_backward(dy, x, w, mean, rstd, dw, None, accumulate=True)
    assert torch.equal(dw, 2 * first[:, :width]) and torch.equal(db, first[:, width:2 * width])


def test_norm_no_rows(layers):
    (w, b), (dw, db), G, _ = params(gen(5), 3, 0, (6,), (6,))
    x = torch.empty(3, 0, 6, device="cuda")
    y, mean, rstd = layers.layer_norm_forward(x, w, b)
    assert y.shape == x.shape and mean.shape == (3, 0)
    layers.layer_norm_backward(x, x, w, mean, rstd, dw, db, accumulate=True)
    assert (G == -7.0).all()
    assert layers.layer_norm_backward(x, x, w, mean, rstd, dw, db).shape == x.shape
    assert (dw == 0).all() and (db == 0).all()


def test_norm_nan_stays_in_its_row(layers):
    g = gen(6)
    n, rows, width = 2, 6, 90
    x = acts(g, n, rows, width, torch.float32)
    (w, b), _, _, _ = params(g, n, 0, (width,), (width,))
    clean, _, _ = layers.layer_norm_forward(x, w, b)
    x[0, 2, 5], x[1, 4, 89] = float("nan"), float("inf")
    y, _, _ = layers.layer_norm_forward(x, w, b)
    bad = torch.zeros(n, rows, dtype=torch.bool, device="cuda")
    bad[0, 2] = bad[1, 4] = True
    assert not torch.isfinite(y[bad]).any()
    assert torch.equal(y[~bad], clean[~bad])


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------
FFN_SIZES = [(1, 1, 1, 1), (2, 3, 5, 7), (4, 1, 96, 130), (3, 17, 33, 65), (2, 8, 31, 40), (1, 129, 257, 31), (2, 128, 64, 128), (2, 130, 64, 171),
             (1, 127, 129, 260), (2, 200, 40, 300), (33, 2, 20, 12), (2, 64, 100, 96), (1, 33, 200, 129)]


def run_ffn(layers, x, dy, p, grads, act):
    y, saved = layers.gated_ffn_forward(x, *p, act, save=True)
    dx = layers.gated_ffn_backward(dy, x, *p, saved, *grads, act)
    return {"y": y, "dx": dx, "dgate": grads[0], "dup": grads[1], "ddown": grads[2]}


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,hidden", FFN_SIZES)
def test_ffn(layers, n, rows, width, hidden, dtype, act):
    g = gen(n, rows, width, hidden)
    x, dy = acts(g, n, rows, width, dtype), acts(g, n, rows, width, dtype)
    p, grads, G, D = params(g, n, 3, (hidden, width), (hidden, width), (width, hidden), spread=0.3)
    got = run_ffn(layers, x, dy, p, grads, act)
    want = ref.gated_ffn(x, *p, act, dy)
    for name in want:
        ref.check(got[name], want[name], f"{name} of {n}x{rows}x{width}x{hidden}")
    untouched(G, 3, D - 3)
    y, none = layers.gated_ffn_forward(x, *p, act)  # prediction: the same y
    assert none is None and torch.equal(y, got["y"])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", ["gap", "rows_first", "shared"])
@pytest.mark.parametrize("n,rows,width,hidden", [(3, 40, 72, 96), (2, 5, 130, 45), (2, 140, 128, 128)])
def test_ffn_layouts(layers, n, rows, width, hidden, layout, dtype):
    g = gen(n, rows, width, hidden, 1)
    x, dy = acts(g, n, rows, width, dtype, layout), acts(g, n, rows, width, dtype, layout)
    p, grads, _, _ = params(g, n, 32, (hidden, width), (hidden, width), (width, hidden), spread=0.2)
    got, want = run_ffn(layers, x, dy, p, grads, "silu"), ref.gated_ffn(x, *p, "silu", dy)
    for name in want:
        ref.check(got[name], want[name], name)


def test_ffn_large_gates(layers):
    """Activations far out on both sides: exp overflows where the sigmoid is 0."""
    g = gen(7)
    n, rows, width, hidden = 2, 20, 32, 48
    x, dy = acts(g, n, rows, width, torch.float32, scale=30.0), acts(g, n, rows, width, torch.float32)
    for act in ("silu", "gelu"):
        p, grads, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
        got, want = run_ffn(layers, x, dy, p, grads, act), ref.gated_ffn(x, *p, act, dy)
        for name in want:
            ref.check(got[name], want[name], f"{act} {name}")


def test_ffn_parts_and_accumulate(layers):
    g = gen(8)
    n, rows, width, hidden = 2, 70, 36, 50
    x, dy = acts(g, n, rows, width, torch.float32), acts(g, n, rows, width, torch.float32)
    p, grads, G, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    dx = layers.gated_ffn_backward(dy, x, *p, saved, *grads)
    first = G.clone()
    assert torch.equal(layers.gated_ffn_backward(dy, x, *p, saved), dx)
    assert torch.equal(G, first)
    for k in range(3):
        G.fill_(-7.0)
        one = [grads[i] if i == k else None for i in range(3)]
        assert layers.gated_ffn_backward(dy, x, *p, saved, *one, want_dx=False) is None
        for i in range(3):
            at = i * hidden * width
            same = first[:, at:at + hidden * width] if i == k else torch.full((n, hidden * width), -7.0, device="cuda")
            assert torch.equal(G[:, at:at + hidden * width], same)
    G.copy_(first)
    layers.gated_ffn_backward(dy, x, *p, saved, *grads, accumulate=True)
    assert torch.equal(G[:, :3 * hidden * width], 2 * first[:, :3 * hidden * width])


def test_ffn_no_rows(layers):
    p, grads, G, _ = params(gen(9), 2, 0, (6, 4), (6, 4), (4, 6))
    x = torch.empty(2, 0, 4, device="cuda", dtype=torch.bfloat16)
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    assert y.shape == x.shape
    layers.gated_ffn_backward(x, x, *p, saved, *grads, accumulate=True)
    assert (G == -7.0).all()
    layers.gated_ffn_backward(x, x, *p, saved, *grads)
    assert all((v == 0).all() for v in grads)


@pytest.mark.parametrize("rows", [2, 40, 150])
def test_ffn_nan_stays_in_its_row(layers, rows):
    g = gen(10)
    n, width, hidden = 2, 40, 50
    x = acts(g, n, rows, width, torch.float32)
    p, _, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    clean, _ = layers.gated_ffn_forward(x, *p)
    x[0, 1, 3], x[1, 0, 39] = float("nan"), float("inf")
    y, _ = layers.gated_ffn_forward(x, *p)
    bad = torch.zeros(n, rows, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 0] = True
    assert not torch.isfinite(y[bad]).any()
    assert torch.equal(y[~bad], clean[~bad])


def test_ffn_same_bits_every_time(layers):
    g = gen(11)
    x, dy = acts(g, 2, 1_000, 96, torch.bfloat16), acts(g, 2, 1_000, 96, torch.bfloat16)
    p, grads, G, _ = params(g, 2, 0, (160, 96), (160, 96), (96, 160))
    a = {k: v.clone() for k, v in run_ffn(layers, x, dy, p, grads, "silu").items()}
    G.fill_(-7.0)
    b = run_ffn(layers, x, dy, p, grads, "silu")
    assert all(torch.equal(a[k], b[k]) for k in a)


# ---------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", ["dense", "gap", "rows_first", "shared"])
@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (2, 3, 5), (3, 7, 33), (2, 20, 64)])
def test_dropout(layers, n, rows, width, layout, dtype):
    g = gen(n, rows, width, 2)
    x, residual = acts(g, n, rows, width, dtype, layout), acts(g, n, rows, width, dtype, layout)
    for p, seed, call in ((0.3, 5, 0), (0.5, -1, 7), (0.0, 1, 2 ** 64 - 1), (1.0, 2, 3)):
        keep = ref.kept(n * rows * width, p, seed, call).view(n, rows, width)
        scaled = x.double().cpu() / (1.0 - p) if p < 1 else torch.zeros(n, rows, width, dtype=torch.float64)
        y = torch.where(keep, scaled, 0.0)
        r = ref.rounding(dtype)
        got = layers.dropout_forward(x, p, seed, call)
        assert torch.equal((got != 0).cpu(), keep & (x != 0).cpu())
        ref.check(got, (y, (r + 3 * ref.U) * y.abs()), "y")
        total = y + residual.double().cpu()
        ref.check(layers.dropout_forward(x, p, seed, call, residual), (total, r * total.abs() + 3 * ref.U * (y.abs() + total.abs())), "y + residual")
        assert torch.equal(layers.dropout_backward(x, p, seed, call), got)


def test_dropout_drops_what_is_not_finite(layers):
    x = torch.full((1, 1, 999), float("nan"), device="cuda")
    keep = ref.kept(999, 0.4, 11, 0)
    assert torch.equal(torch.isnan(layers.dropout_forward(x, 0.4, 11))[0, 0].cpu(), keep)
    x.fill_(float("inf"))
    assert torch.equal(torch.isinf(layers.dropout_forward(x, 0.4, 11))[0, 0].cpu(), keep)
    assert (layers.dropout_forward(x, 1.0, 11) == 0).all()


def test_dropout_far_indices(layers):
    """More than 2^32 values: the bits of those behind are those of their own index."""
    n, rows, width = 2, 1, (1 << 31) + 50
    x = torch.ones(n, rows, width, dtype=torch.bfloat16, device="cuda")
    y = layers.dropout_forward(x, 0.5, 13)
    del x
    for start in (0, (1 << 31) - 50, (1 << 32) - 10, 2 * width - 100):
        assert torch.equal((y.view(-1)[start:start + 100] != 0).cpu(), ref.kept(100, 0.5, 13, 0, start=start)), start


def test_dropout_rate(layers):
    """Of a million values about a tenth is dropped: within five standard deviations."""
    y = layers.dropout_forward(torch.ones(1, 1000, 1000, device="cuda"), 0.1, 99)
    assert abs((y == 0).sum().item() - 100_000) < 5 * 300


def test_dropout_counter(layers):
    x = torch.randn(2, 3, 50, device="cuda")
    counter = torch.tensor([41], dtype=torch.int64, device="cuda")
    a = layers.dropout_forward(x, 0.5, 3, 1, counter=counter)
    assert torch.equal((a != 0).view(-1).cpu(), ref.kept(300, 0.5, 3, 1, counter=41))
    counter += 1
    b = layers.dropout_forward(x, 0.5, 3, 1, counter=counter)
    assert torch.equal((b != 0).view(-1).cpu(), ref.kept(300, 0.5, 3, 1, counter=42))


# ---------------------------------------------------------------------------------------------
# how they are called
# ---------------------------------------------------------------------------------------------
def test_more_dimensions(layers):
    g = gen(12)
    x = acts(g, 2, 12, 20, torch.float32)
    x5, x2 = x.view(2, 3, 2, 2, 20), x[:, 0]
    p, _, _, _ = params(g, 2, 0, (30, 20), (30, 20), (20, 30))
    (w, b), _, _, _ = params(g, 2, 0, (20,), (20,))
    for f in (lambda t: layers.gated_ffn_forward(t, *p)[0], lambda t: layers.layer_norm_forward(t, w, b)[0], lambda t: layers.dropout_forward(t, 0.3, 1)):
        y = f(x)
        assert torch.equal(f(x5).view(2, 12, 20), y) and f(x5).shape == x5.shape
        assert f(x2).shape == x2.shape
    assert torch.equal(layers.layer_norm_forward(x5.permute(0, 3, 1, 2, 4), w, b)[0], layers.layer_norm_forward(x5, w, b)[0].permute(0, 3, 1, 2, 4))


def test_refusals(layers):
    x = torch.zeros(2, 3, 8, device="cuda")
    w = torch.zeros(2, 8, device="cuda")
    gate, down = torch.zeros(2, 4, 8, device="cuda"), torch.zeros(2, 8, 4, device="cuda")
    y, saved = layers.gated_ffn_forward(x, gate, gate, down, save=True)
    cases = [
        (TypeError, "contiguous rows", lambda: layers.layer_norm_forward(x.transpose(1, 2), torch.zeros(2, 3, device="cuda"))),
        (TypeError, "float32, bfloat16 or float16", lambda: layers.layer_norm_forward(x.double(), w)),
        (TypeError, "x must be", lambda: layers.layer_norm_forward(x[0, 0], w)),
        (ValueError, "weight must have the shape", lambda: layers.layer_norm_forward(x, w[:1])),
        (TypeError, "weight must be a float32", lambda: layers.layer_norm_forward(x, w.bfloat16())),
        (TypeError, "weight must be a float32", lambda: layers.layer_norm_forward(x, w.cpu())),
        (TypeError, "contiguous within", lambda: layers.layer_norm_forward(x, torch.zeros(2, 16, device="cuda")[:, ::2])),
        (ValueError, "dy must have", lambda: layers.layer_norm_backward(x.bfloat16(), x, w, w[:, :3], w[:, :3])),
        (TypeError, "mean must be", lambda: layers.layer_norm_backward(x, x, w, w, w)),
        (ValueError, "activation must be", lambda: layers.gated_ffn_forward(x, gate, gate, down, "relu")),
        (ValueError, "up must have the shape", lambda: layers.gated_ffn_forward(x, gate, down, down)),
        (TypeError, "saved must be", lambda: layers.gated_ffn_backward(x, x, gate, gate, down, None)),
        (TypeError, "saved must be", lambda: layers.gated_ffn_backward(x, x, gate, gate, down, saved[1:])),
        (ValueError, "residual must have", lambda: layers.dropout_forward(x, 0.5, 1, residual=x[:, :2])),
        (TypeError, "counter must be", lambda: layers.dropout_forward(x, 0.5, 1, counter=torch.zeros(1, device="cuda"))),
        (layers.SvgdError, "INVALID_ARG", lambda: layers.dropout_forward(x, 1.5, 1)),
        (layers.SvgdError, "INVALID_ARG", lambda: layers.layer_norm_forward(x, w, eps=float("nan"))),
        (layers.SvgdError, "TOO_LARGE", lambda: layers.layer_norm_forward(torch.zeros(1, 1, 16385, device="cuda"), torch.zeros(1, 16385, device="cuda"))),
        (layers.SvgdError, "TOO_LARGE", lambda: layers.dropout_forward(torch.zeros(65, 1, 1, device="cuda"), 0.5, 1)),
        # a gradient that is written where the parameters are, or two in one place
        (layers.SvgdError, "INVALID_ARG", lambda: layers.gated_ffn_backward(x, x, gate, gate, down, saved, gate)),
        (layers.SvgdError, "INVALID_ARG", lambda: layers.layer_norm_backward(x, x, w, *torch.zeros(2, 2, 3, device="cuda"), *[torch.zeros(2, 8, device="cuda")] * 2)),
    ]
    for error, words, call in cases:
        with pytest.raises(error, match=words):
            call()
    torch.cuda.synchronize()


def test_another_stream(layers):
    """A call on a stream that is not the current one waits for what that stream has to do first."""
    g = gen(13)
    n, rows, width, hidden = 2, 300, 64, 96
    x = acts(g, n, rows, width, torch.float32)
    p, grads, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    dx = layers.gated_ffn_backward(x, x, *p, saved, *grads)
    want = [t.clone() for t in (y, dx, *grads)]
    side = torch.cuda.Stream()
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.randn(1 << 22, device="cuda").sort()
        late.copy_(x)
    y, saved = layers.gated_ffn_forward(late, *p, save=True, stream=side)
    dx = layers.gated_ffn_backward(late, late, *p, saved, *grads, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, *grads), want))


def test_captured_and_replayed(layers):
    """Forward and backward of all three in one graph, replayed on new inputs between eager work; the counter moves on."""
    g = gen(14)
    n, rows, width, hidden = 2, 90, 48, 80
    x, dy = acts(g, n, rows, width, torch.float32), acts(g, n, rows, width, torch.float32)
    (w, b), (dw, db), _, _ = params(g, n, 0, (width,), (width,))
    p, grads, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        h, mean, rstd = layers.layer_norm_forward(x, w, b)
        z, saved = layers.gated_ffn_forward(h, *p, save=True)
        s = layers.dropout_forward(z, 0.2, 17, 0, x, counter)
        dz = layers.dropout_backward(dy, 0.2, 17, 0, counter)
        dh = layers.gated_ffn_backward(dz, h, *p, saved, *grads)
        return s, layers.layer_norm_backward(dh, x, w, mean, rstd, dw, db)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(torch.randn(x.shape, generator=g).cuda())
        counter.fill_(k)
        want = [t.clone() for t in (*step(), dw, db, *grads)]
        torch.cuda.synchronize()
        for t in (dw, db, *grads):
            t.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, dw, db, *grads), want)), k


# ---------------------------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------------------------
def test_autograd_matches_the_plain_calls(layers):
    g = gen(15)
    n, rows, width, hidden = 2, 30, 24, 40
    x, dy = acts(g, n, rows, width, torch.bfloat16), acts(g, n, rows, width, torch.bfloat16)
    (w, b), (dw, db), _, _ = params(g, n, 0, (width,), (width,))
    p, grads, G, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    h, mean, rstd = layers.layer_norm_forward(x, w, b)
    z, saved = layers.gated_ffn_forward(h, *p, "gelu", save=True)
    s = layers.dropout_forward(z, 0.2, 17, 5, x)
    dz = layers.dropout_backward(dy, 0.2, 17, 5)
    dh = layers.gated_ffn_backward(dz, h, *p, saved, *grads, "gelu")
    dx = layers.layer_norm_backward(dh, x, w, mean, rstd, dw, db)

    leaves = [t.detach().requires_grad_() for t in (x, w, b, *p)]
    gw = torch.zeros_like(G)  # the block's gradients land in a matrix like G
    for k, t in enumerate(leaves[3:]):
        t.grad = gw[:, k * hidden * width:(k + 1) * hidden * width].view(t.shape)
    out = layers.dropout(layers.gated_ffn(layers.layer_norm(leaves[0], *leaves[1:3]), *leaves[3:], "gelu"), 0.2, 17, 5, leaves[0])
    assert torch.equal(out, s)
    out.backward(dy)
    assert torch.equal(leaves[1].grad, dw) and torch.equal(leaves[2].grad, db)
    for k, (t, want) in enumerate(zip(leaves[3:], grads)):
        assert torch.equal(t.grad, want) and t.grad.data_ptr() == gw.data_ptr() + 4 * k * hidden * width
    assert torch.equal(leaves[0].grad, dx + dy)  # the branch and the residual stream


def test_autograd_of_a_shared_batch_and_a_sum(layers):
    """A batch that all particles share gets the sum of their gradients; a sum's gradient has no strides."""
    g = gen(16)
    n, rows, width, hidden = 3, 10, 16, 24
    batch = torch.randn(rows, width, generator=g).cuda().requires_grad_()
    p, _, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden))
    layers.gated_ffn(batch.expand(n, -1, -1), *p).sum().backward()
    want = ref.gated_ffn(batch.detach().expand(n, -1, -1), *p, "silu", torch.ones(n, rows, width))["dx"]
    ref.check(batch.grad, (want[0].sum(0), want[1].sum(0) + 4 * ref.U * want[0].abs().sum(0)), "gradient of the batch")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(layers, act):
    """The whole block's gradient along a direction against a central difference of its value: both in fp32, differences of 2e-2 of
    values around 1, a cubic term below 1e-3."""
    g = gen(17)
    n, rows, width, hidden = 2, 12, 20, 28
    x = acts(g, n, rows, width, torch.float32)
    c = acts(g, n, rows, width, torch.float32).double()
    (w, b), _, _, _ = params(g, n, 0, (width,), (width,))
    p, _, _, _ = params(g, n, 0, (hidden, width), (hidden, width), (width, hidden), spread=0.3)
    leaves = [t.detach().clone().requires_grad_() for t in (x, w, b, *p)]

    def value(ts):
        return (layers.dropout(layers.gated_ffn(layers.layer_norm(*ts[:3]), *ts[3:], act), 0.25, 3, 0, ts[0]).double() * c).sum()

    value(leaves).backward()
    for k, leaf in enumerate(leaves):
        d = torch.randn(leaf.shape, generator=g).cuda()
        d /= d.norm()
        t = 1e-2
        sides = [value([q.detach() + (s * t * d if i == k else 0) for i, q in enumerate(leaves)]).item() for s in (1, -1)]
        slope = (leaf.grad.double() * d).sum().item()
        size = (leaf.grad.double() ** 2).sum().sqrt().item()
        assert abs((sides[0] - sides[1]) / (2 * t) - slope) <= 2e-3 * size, k
