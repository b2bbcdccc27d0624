"""The particles' layers where sizes lead the kernels to ways that the other tests' sizes do not."""
import pytest
import torch

import layer_reference as ref
from ffn_shapes import DX_OF_FEW_ROWS, THIN, TILES
from test_gpu_layers import IDS, TYPES, acts, gen, layers, params, run_ffn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_ffn_more_small_tiles_than_a_launch_takes(layers):  # noqa: F811
    """600 million rows of a narrow layer, 77 GB of h: the fastest tiles would be 18.75 million."""
    rows, width, hidden = 600_000_000, 8, 32
    x = torch.rand(1, rows, width, generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16) - 0.5
    p, _, _, _ = params(gen(41), 1, 3, (hidden, width), (hidden, width), (width, hidden), spread=0.5)
    y, _ = layers.gated_ffn_forward(x, *p)
    for first in (0, rows // 2 - 7, (1 << 26) * 8 - 20, rows - 40):  # (the third: where x's values pass 2^32)
        part = slice(first, first + 40)
        ref.check(y[:, part], ref.gated_ffn(x[:, part], *p, "silu")["y"], f"y from row {first} on")


def check_block(layers, n, rows, width, hidden, dtype, act, layout="gap"):  # noqa: F811
    g = gen(n, rows, width, hidden, 5)
    x, dy = acts(g, n, rows, width, dtype, layout), acts(g, n, rows, width, dtype, layout)
    p, grads, G, D = params(g, n, 3, (hidden, width), (hidden, width), (width, hidden), spread=width ** -0.5)
    got, want = run_ffn(layers, x, dy, p, grads, act), ref.gated_ffn(x, *p, act, dy)
    for name in want:
        ref.check(got[name], want[name], f"{name} of {n}x{rows}x{width}x{hidden}")
    assert (G[:, :3] == -7.0).all() and (G[:, D - 3:] == -7.0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,hidden", THIN)
def test_ffn_few_rows_of_several_steps(layers, n, rows, width, hidden, dtype):  # noqa: F811
    check_block(layers, n, rows, width, hidden, dtype, "gelu")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,hidden", TILES)
def test_ffn_tiles_of_several_steps(layers, n, rows, width, hidden, dtype):  # noqa: F811
    check_block(layers, n, rows, width, hidden, dtype, "silu")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,rows,width,hidden", [(1, 3, 5, 1 << 20), (1, 35, 3, 1 << 20), (1, 3, 1 << 20, 4), (1, 70, (1 << 20) - 3, 5)])
def test_ffn_as_wide_as_may_be(layers, n, rows, width, hidden, dtype):  # noqa: F811
    check_block(layers, n, rows, width, hidden, dtype, "silu")


def far_rows(g, n, rows, width, dtype):
    """Rows (1 << 22) + 57 values apart, the particles' side by side."""
    stride = (1 << 22) + 57
    assert n * (width + 2) <= stride
    buf = torch.empty(rows * stride, dtype=dtype, device="cuda")
    return buf.as_strided((n, rows, width), (width + 2, stride, 1), 1).copy_(torch.randn(n, rows, width, generator=g).to(dtype).cuda())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows", [7, 70, 260])
def test_rows_far_apart(layers, rows, dtype):  # noqa: F811
    n, width, hidden = 2, 109, 131
    g = gen(rows, 6)
    x, dy = far_rows(g, n, rows, width, dtype), far_rows(g, n, rows, width, dtype)
    p, grads, _, _ = params(g, n, 3, (hidden, width), (hidden, width), (width, hidden), spread=0.2)
    got, want = run_ffn(layers, x, dy, p, grads, "silu"), ref.gated_ffn(x, *p, "silu", dy)
    for name in want:
        ref.check(got[name], want[name], name)
    (w, b), (dw, db), _, _ = params(g, n, 1, (width,), (width,))
    y, mean, rstd = layers.layer_norm_forward(x, w, b)
    got = {"y": y, "dx": layers.layer_norm_backward(dy, x, w, mean, rstd, dw, db), "dweight": dw, "dbias": db}
    want = ref.layer_norm(x, w, b, 1e-5, dy)
    for name in got:
        ref.check(got[name], want[name], name)
    assert torch.equal(layers.dropout_forward(x, 0.3, 5, residual=dy), layers.dropout_forward(x.contiguous(), 0.3, 5, residual=dy.contiguous()))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,width,hidden", DX_OF_FEW_ROWS)
def test_ffn_gradients_of_few_rows(layers, n, rows, width, hidden, dtype):  # noqa: F811
    """All gradients, dx alone, and the parameters' alone."""
    g = gen(n, rows, width, hidden, 7)
    x, dy = acts(g, n, rows, width, dtype, "gap"), acts(g, n, rows, width, dtype)
    p, grads, G, D = params(g, n, 3, (hidden, width), (hidden, width), (width, hidden), spread=width ** -0.5)
    want = ref.gated_ffn(x, *p, "silu", dy)
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    dx = layers.gated_ffn_backward(dy, x, *p, saved, *grads)
    for name, got in (("y", y), ("dx", dx), ("dgate", grads[0]), ("dup", grads[1]), ("ddown", grads[2])):
        ref.check(got, want[name], name)
    first = [t.clone() for t in grads]
    ref.check(layers.gated_ffn_backward(dy, x, *p, saved), want["dx"], "dx alone")
    assert torch.equal(layers.gated_ffn_backward(dy, x, *p, saved, None, grads[1], None, accumulate=True), dx)
    assert torch.equal(grads[0], first[0]) and torch.equal(grads[1], 2 * first[1]) and torch.equal(grads[2], first[2])
    assert layers.gated_ffn_backward(dy, x, *p, saved, *grads, want_dx=False) is None
    assert all(torch.equal(a, b) for a, b in zip(grads, first))
    assert (G[:, :3] == -7.0).all() and (G[:, D - 3:] == -7.0).all()


def test_ffn_no_rows_of_many_particles(layers):  # noqa: F811
    p, grads, G, _ = params(gen(42), 40, 0, (400, 300), (400, 300), (300, 400))
    x = torch.empty(40, 0, 300, device="cuda")
    y, saved = layers.gated_ffn_forward(x, *p, save=True)
    assert layers.gated_ffn_backward(x, x, *p, saved, *grads, accumulate=True).shape == x.shape
    assert (G == -7.0).all()
    layers.gated_ffn_backward(x, x, *p, saved, *grads)
    assert all((v == 0).all() for v in grads)
