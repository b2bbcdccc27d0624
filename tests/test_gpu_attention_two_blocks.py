"""Attention of so many workgroups that a wave has two blocks of rows or of keys: every instance that has them, unmasked, causal and with every mask, some sequences against the definitions.
test_attention_rules.py holds that these sizes lead there."""
import pytest
import torch

import attention_reference as ref
from test_gpu_attention import IDS, TYPES, gen, masks_of

pytestmark = pytest.mark.gpu

# n, batch, tokens, keys, heads, kv_heads, dim
UNMASKED = [(16, 16, 130, 130, 8, 8, 5), (16, 16, 130, 130, 8, 8, 24), (24, 16, 135, 150, 12, 4, 64), (16, 16, 70, 130, 8, 8, 90), (16, 16, 66, 66, 8, 8, 120)]
CAUSAL = [(32, 32, 66, 66, 2, 2, 5), (16, 16, 130, 130, 8, 8, 24), (16, 16, 140, 130, 8, 8, 64), (16, 20, 70, 200, 8, 8, 90), (16, 12, 140, 140, 8, 8, 120)]
LONG = [(2, 4, 2_050, 2_060, 8, 8, d) for d in (7, 32, 50, 96, 128)]  # (masked calls of fewer workgroups)
KINDS = ["lengths", "ragged", "starts", "prefix", "documents", "mixed_documents", "everything"]
MASKED = [(10, 15, 140, 150, 10, 10, 24), (10, 15, 141, 160, 10, 10, 64), (10, 15, 70, 180, 30, 15, 90), (10, 15, 140, 140, 10, 10, 120)]


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def run(att, n, batch, t, s, heads, kv, d, dtype, how, places):
    """places: particle, sequence, key head"""
    g = torch.Generator(device="cuda").manual_seed(t + d)
    make = lambda tokens, h: torch.randn(n, batch, tokens, h, d, generator=g, device="cuda").to(dtype)  # noqa: E731
    q, do, k, v = make(t, heads), make(t, heads), make(s, kv), make(s, kv)
    if "lengths" in how:  # what lies behind is not read
        for b, m in enumerate(how["lengths"].tolist()):
            k[:, b, max(0, m):] = float("nan")
            v[:, b, max(0, m):] = float("inf")
    o, lse = att.attention_forward(q, k, v, **how)
    got = dict(zip(("o", "dq", "dk", "dv"), (o, *att.attention_backward(do, q, k, v, o, lse, **how))))
    group = heads // kv
    for i, b, h in places:
        rows, keys = (lambda x: x[i:i + 1, b:b + 1, :, h * group:(h + 1) * group]), (lambda x: x[i:i + 1, b:b + 1, :, h:h + 1])
        want = ref.attention(rows(q), keys(k), keys(v), rows(do), **{x: m[b:b + 1] if torch.is_tensor(m) else m for x, m in how.items()})
        for name, x in got.items():
            ref.check((keys if name in ("dk", "dv") else rows)(x), want[name], f"{name} of {i}, {b}, {h}")
        ref.check_lse(lse[i:i + 1, b:b + 1, h * group:(h + 1) * group], want["lse"])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", UNMASKED, ids=str)
def test_unmasked(att, size, dtype):
    n, batch, _, _, _, kv, _ = size
    run(att, *size, dtype, {}, [(0, 0, 0), (n - 1, batch - 1, kv - 1), (n // 2, 3, kv // 2)])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", CAUSAL, ids=str)
def test_causal(att, size, dtype):
    n, batch, _, _, _, kv, _ = size
    run(att, *size, dtype, {"causal": True}, [(0, 0, 0), (n - 1, batch - 1, kv - 1), (n // 2, 3, kv // 2)])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", LONG, ids=str)
def test_long_causal(att, size, dtype):
    run(att, *size, dtype, {"causal": True}, [(1, 2, 5)])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", MASKED, ids=str)
def test_masks(att, size, kind, dtype):
    n, batch, t, s, _, kv, _ = size
    how = masks_of(kind, gen(t, s, kind, "two"), batch, t, s)
    run(att, *size, dtype, how, [(b % n, b, (3 * b) % kv) for b in (0, 1, 2, 3, 4)])  # (masks_of has five kinds of a mask, by turns)
