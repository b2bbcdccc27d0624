"""Scales and caps at the ends of what fp32 holds: refused where the kernels cannot form what they need of them (CPU), right up to there (GPU)."""
import pytest
import torch

from test_attention_cpu import INVALID, attention_backward, attention_forward, lib  # noqa: F401


@pytest.mark.parametrize("bad", [dict(cap=2.4e38), dict(cap=3.4e38), dict(scale=2.4e38), dict(scale=0.1, cap=1e38), dict(scale=1e-30, cap=1e16), dict(scale=1e-30, cap=1e8), dict(scale=1e9, cap=1e-30),
                                 dict(scale=3e38, cap=3e38)])
def test_what_fp32_cannot_form_is_refused(lib, bad):  # noqa: F811
    assert attention_forward(lib, **bad) == INVALID
    assert attention_backward(lib, **bad) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("t,s", [(40, 70), (2, 300)])
def test_caps_that_cap_nothing(dtype, t, s):
    """tanh of what is far below 1 is that itself: the same results as without a cap, but for two more roundings of scores below 2^4 in exponents (2^-23 2^5 of a probability, a few times that of a gradient), and at most
    a step of the type where that crosses a rounding's border."""
    from paper_2306_06528_amd import attention as att
    g = torch.Generator().manual_seed(s)
    q, do = ((torch.randn(1, 2, t, 4, 64, generator=g)).to(dtype).cuda() for _ in range(2))
    k, v = ((torch.randn(1, 2, s, 2, 64, generator=g)).to(dtype).cuda() for _ in range(2))
    run = lambda **how: (lambda o, lse: (o, *att.attention_backward(do, q, k, v, o, lse, **how)))(*att.attention_forward(q, k, v, **how))  # noqa: E731
    for plain, cap in (({}, 1e36), ({}, 1e30), ({"scale": 1e-3}, 1e34)):
        for got, want in zip(run(cap=cap, **plain), run(**plain)):
            got, want = got.float(), want.float()
            step = 2.0 ** -16 if dtype == torch.float32 else torch.finfo(dtype).eps
            assert ((got - want).abs() <= step * want.abs() + 2.0 ** -16 * want.abs().max()).all(), cap
