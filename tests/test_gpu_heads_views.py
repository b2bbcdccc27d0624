"""Outputs with heads that are views of one buffer, as the C ABI takes them: dq, dk and dv (or q and k) side by side in every token, with something between and behind them that stays as it was."""
import ctypes

import pytest
import torch

from test_attention_cpu import Attention, Heads, Rotary, lib  # noqa: F401
from test_gpu_attention import gen, normal, params

pytestmark = pytest.mark.gpu
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
IDS = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def heads(t):
    return Heads(t.data_ptr(), *t.stride()[:4])


def buffer(n, batch, t, total, d, dtype, order):
    """(n, batch, tokens, heads, dim) with the tokens or the heads outside, filled with a value that is to stay."""
    shape = (n, batch, t, total, d) if order == "tokens" else (n, total, batch, t, d)
    buf = torch.full(shape, -7.0, dtype=dtype, device="cuda")
    return buf if order == "tokens" else buf.permute(0, 2, 3, 1, 4)


@pytest.mark.parametrize("order", ["tokens", "heads"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_gradients_of_one_buffer(att, lib, dtype, order):  # noqa: F811
    n, batch, t, h, kv, d = 2, 2, 70, 4, 2, 40
    g = gen("views", order)
    qkv = normal(g, n, batch, t, h + 2 * kv, d, dtype=dtype)
    q, k, v = qkv[..., :h, :], qkv[..., h:h + kv, :], qkv[..., h + kv:, :]
    do = normal(g, n, batch, t, h, d, dtype=dtype)
    o, lse = att.attention_forward(q, k, v, causal=True)
    want = att.attention_backward(do, q, k, v, o, lse, causal=True)
    dqkv = buffer(n, batch, t, h + 2 * kv + 2, d, dtype, order)
    dq, dk, dv = dqkv[..., :h, :], dqkv[..., h + 1:h + 1 + kv, :], dqkv[..., h + 1 + kv:-1, :]
    a = Attention(n, h, kv, d, batch, t, t, 1, d ** -0.5, 0.0, None, 0, None, None, None, None)
    size = lib.svgd_attention_scratch(ctypes.byref(a))
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call(dk):
        return lib.svgd_attention_backward(DTYPES[dtype], ctypes.byref(a), heads(do), heads(q), heads(k), heads(v), heads(o), lse.data_ptr(), heads(dq), heads(dk), heads(dv), None, 0, 0,
                                           scratch.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    assert call(dqkv[..., h - 1:h - 1 + kv, :]) == -1  # (a head of dq's)
    torch.cuda.synchronize()
    assert (dqkv == -7.0).all()
    assert call(dk) == 0
    for got, x in zip((dq, dk, dv), want):
        assert torch.equal(got, x)
    assert (dqkv[..., h, :] == -7.0).all() and (dqkv[..., -1, :] == -7.0).all()


@pytest.mark.parametrize("order", ["tokens", "heads"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_results_of_one_buffer(att, lib, dtype, order):  # noqa: F811
    """Rotated queries and keys beside each other, and o beside them; the gradients likewise."""
    n, batch, t, h, kv, d = 2, 2, 21, 3, 1, 24
    g = gen("rotary views", order)
    q, k, v, dq, dk = (normal(g, n, batch, t, x, d, dtype=dtype) for x in (h, kv, kv, h, kv))
    (qw, kw), (dqw, dkw), G, _ = params(g, n, 0, (d,), (d,))
    frequencies = torch.tensor([0.5 ** j for j in range(d // 2)], dtype=torch.float64, device="cuda")
    positions = torch.arange(t, device="cuda")
    how = {"frequencies": frequencies, "positions": positions}
    r = Rotary(n, h, kv, d, d // 2, 0, batch, t, frequencies.data_ptr(), positions.data_ptr(), 0, 1e-6, qw.data_ptr(), kw.data_ptr(), qw.stride(0), kw.stride(0))
    stream = torch.cuda.current_stream().cuda_stream
    buf = buffer(n, batch, t, 2 * h + kv, d, dtype, order)
    q_out, k_out, o_out = buf[..., :h, :], buf[..., h:h + kv, :], buf[..., h + kv:, :]
    assert lib.svgd_qk_norm_rotary_forward(DTYPES[dtype], ctypes.byref(r), heads(q), heads(k), heads(q_out), heads(buf[..., h - 1:h - 1 + kv, :]), stream) == -1
    assert lib.svgd_qk_norm_rotary_forward(DTYPES[dtype], ctypes.byref(r), heads(q), heads(k), heads(q_out), heads(k_out), stream) == 0
    for got, x in zip((q_out, k_out), att.qk_norm_rotary_forward(q, k, qw, kw, **how)):
        assert torch.equal(got, x)
    assert (o_out == -7.0).all()
    a = Attention(n, h, kv, d, batch, t, t, 1, d ** -0.5, 0.0, None, 0, None, None, None, None)
    assert lib.svgd_attention_forward_scratch(ctypes.byref(a)) == 0
    assert lib.svgd_attention_forward(DTYPES[dtype], ctypes.byref(a), heads(q_out), heads(k_out), heads(v), heads(o_out), None, None, 0, stream) == 0
    assert torch.equal(o_out, att.attention_forward(q_out, k_out, v, causal=True)[0])
    want = att.qk_norm_rotary_backward(dq, dk, q, k, qw, kw, dqw, dkw, **how)
    weights = G.clone()
    buf = buffer(n, batch, t, h + kv + 1, d, dtype, order)
    size = lib.svgd_qk_norm_rotary_scratch(ctypes.byref(r))
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    G.fill_(-7.0)
    assert lib.svgd_qk_norm_rotary_backward(DTYPES[dtype], ctypes.byref(r), heads(dq), heads(dk), heads(q), heads(k), heads(buf[..., :h, :]), heads(buf[..., h:h + kv, :]), dqw.data_ptr(),
                                            dqw.stride(0), dkw.data_ptr(), dkw.stride(0), 0, scratch.data_ptr(), size, stream) == 0
    assert torch.equal(buf[..., :h, :], want[0]) and torch.equal(buf[..., h:h + kv, :], want[1]) and (buf[..., -1, :] == -7.0).all() and torch.equal(G, weights)
