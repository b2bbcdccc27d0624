"""The attention half where sizes and strides lead the kernels to ways that the other tests' do not."""
import pytest
import torch

import attention_reference as ref
from test_gpu_attention import IDS, TYPES, gen, normal, params
from test_gpu_layers_reach import far_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("rows", [7, 31, 70, 260])
def test_linear_of_rows_far_apart(att, rows, act, dtype):
    """Rows more than 2^22 values apart: offsets within a tile would not fit 32 bits.  Without an activation the products read dy where it is."""
    n, width, out = 2, 109, 131
    g = gen(rows, act, "far")
    x, dy, residual = far_rows(g, n, rows, width, dtype), far_rows(g, n, rows, out, dtype), far_rows(g, n, rows, out, dtype)
    (w, b), (dw, db), G, D = params(g, n, 3, (out, width), (out,), spread=0.2)
    y, saved = att.linear_forward(x, w, b, act, residual, save=True)
    dx = att.linear_backward(dy, x, w, saved, dw, db, act)
    want = ref.linear(x, w, b, act, residual, dy)
    for name, got in (("y", y), ("dx", dx), ("dweight", dw), ("dbias", db)):
        ref.check(got, want[name], name)
    assert (G[:, :3] == -7.0).all() and (G[:, D - 3:] == -7.0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("batch,t", [(300, 1), (90, 3)])
def test_rotary_of_short_sequences(att, batch, t, dtype):
    """One head of few values: a team goes on by 64 heads at a time, which are as many sequences of one token."""
    n, d = 2, 8
    g = gen(batch, t)
    q, k, dq, dk = (normal(g, n, batch, t, 1, d, dtype=dtype) for _ in range(4))
    (qw, kw), (dqw, dkw), G, D = params(g, n, 1, (d,), (d,))
    how = {"frequencies": torch.tensor([1.0, 0.25, 0.1], dtype=torch.float64, device="cuda"), "positions": torch.randint(0, 1_000, (batch, t), generator=g).cuda(), "layout": "half", "eps": 1e-6}
    got = dict(zip(("q", "k"), att.qk_norm_rotary_forward(q, k, qw, kw, **how)))
    got |= dict(zip(("dq", "dk"), att.qk_norm_rotary_backward(dq, dk, q, k, qw, kw, dqw, dkw, **how)))
    for name, x, w, dy, dw in (("q", q, qw, dq, dqw), ("k", k, kw, dk, dkw)):
        want = ref.qk_norm_rotary(x, w, how["frequencies"], how["positions"], "half", 1e-6, dy)
        ref.check(got[name], want["y"], name)
        ref.check(got["d" + name], want["dx"], "d" + name)
        ref.check(dw, want["dweight"], f"d{name}_weight")
    assert (G[:, :1] == -7.0).all() and (G[:, D - 3:] == -7.0).all()
