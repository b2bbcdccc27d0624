"""Attention of 16-bit activations holds in fp32 what it sums up: o, dq, dk and dv are off from the exact result, in the root mean square, by what rounding that result does.

How near to 1 the ratio has to be: what an output is rounded to is off by step / sqrt(12) where the value is in its binade, 2^-9.3 (bf16) or 2^-12.3 (fp16) of it on an average.  What comes before, the fp32 sums,
exponents of at most 2^5 or so (2^-24 2^5 of a probability) and operands in two parts (2^-17 of bf16, 2^-22 of fp16), is below 2^-16.3 of the values, a sixteenth of that and mostly independent of it: the
ratio is below sqrt(1 + 2^-8) = 1.002.  A tenth more of that, for gradients whose terms cancel to a third: sqrt(1 + 9 2^-8) = 1.018.  An operand in one part alone is off by as much as the result's rounding and
makes it 1.4 where a row sees few keys."""
import zlib

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
IDS = ["bf16", "f16"]
MOST = 1.018


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def normal(key, *shape, dtype):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def documents(tokens, batch, s):
    """Documents of so many tokens one behind the other, whose ends do not meet those of tiles."""
    return (torch.arange(s, dtype=torch.int32)[None].expand(batch, s) // tokens).contiguous().cuda()


def ratio(got, exact):
    exact = exact.double()
    rounded = exact.to(got.dtype).double()
    return ((got.double().cpu() - exact).square().mean() / (rounded - exact).square().mean()).sqrt().item()


CASES = {  # n, batch, tokens, keys, heads, kv_heads, dim, how
    "unmasked": (1, 2, 200, 200, 4, 4, 64, {}),
    "few_keys": (2, 4, 40, 40, 4, 4, 64, {}),
    "causal": (1, 1, 512, 512, 4, 2, 64, {"causal": True}),
    "documents_of_32": (1, 2, 512, 512, 2, 2, 64, {"causal": True, "documents": 32}),
    "documents_of_8": (1, 2, 509, 509, 2, 1, 128, {"documents": 8}),
    "documents_of_3": (1, 2, 512, 512, 2, 2, 64, {"documents": 3}),
    "documents_in_parts": (1, 1, 1_700, 1_700, 2, 1, 32, {"causal": True, "documents": 7}),
    "documents_and_cap": (1, 2, 300, 300, 4, 2, 96, {"documents": 5, "cap": 4.0}),
    "steep_slopes": (1, 1, 512, 512, 4, 4, 128, {"causal": True, "slopes": 2.0}),
    "slopes_and_cap": (1, 2, 320, 320, 4, 2, 72, {"causal": True, "slopes": 1.0, "cap": 6.0}),
    "many_workgroups": (16, 16, 200, 200, 4, 4, 64, {}),
    "few_rows": (4, 2, 2, 700, 8, 2, 64, {"causal": True}),
    "cache": (4, 4, 1, 4_096, 8, 2, 128, {}),
}


def run(att, name, dtype):
    """How far each result is off, over what rounding the exact one is."""
    n, batch, t, s, heads, kv, d, how = CASES[name]
    q, do = (normal((name, x), n, batch, t, heads, d, dtype=dtype) for x in "qd")
    k, v = (normal((name, x), n, batch, s, kv, d, dtype=dtype) for x in "kv")
    how = dict(how)
    if "documents" in how:
        how["documents"] = documents(how["documents"], batch, s)
    if "slopes" in how:
        how["slopes"] = (how["slopes"] * 2.0 ** -torch.arange(heads).float()).repeat(n, 1).cuda()
    o, lse = att.attention_forward(q, k, v, **how)
    got = dict(zip(("o", "dq", "dk", "dv"), (o, *att.attention_backward(do, q, k, v, o, lse, **how))))
    part = lambda x: x[:1, :2] if n > 4 else x  # noqa: E731  (as many as the exact results take seconds for)
    want = ref.attention(part(q), part(k), part(v), part(do), **how)
    off = {x: ratio(part(got[x]), want[x][0]) for x in got}
    print(name, {x: round(r, 4) for x, r in off.items()})
    return off


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("name", CASES)
def test_sums_of_probabilities(att, name, dtype):
    off = run(att, name, dtype)
    assert off["o"] <= MOST and off["dv"] <= MOST, off


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("name", CASES)
def test_gradients_of_scores(att, name, dtype):
    """Rows that see few keys, or few that count: what o's rounding leaves delta off by is not in dq and dk."""
    off = run(att, name, dtype)
    assert off["dq"] <= MOST and off["dk"] <= MOST, off


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("documents_of", [7, 1])
def test_keys_alone(att, documents_of, dtype):
    """dk and dv are the same whether dq is wanted or not, with queries' rows in parts too.  A document of one token: its probability is 1 whatever its score, so dq and dk are 0 but for fp32's roundings of dP - delta,
    (d + 8) 2^-24 of sum |do v|, times the other operand."""
    n, batch, t, heads, kv, d = 1, 1, 1_700, 2, 1, 32
    q, do = (normal(("alone", x), n, batch, t, heads, d, dtype=dtype) for x in "qd")
    k, v = (normal(("alone", x), n, batch, t, kv, d, dtype=dtype) for x in "kv")
    how = {"causal": True, "documents": documents(documents_of, batch, t)}
    o, lse = att.attention_forward(q, k, v, **how)
    dq, dk, dv = att.attention_backward(do, q, k, v, o, lse, **how)
    none, dk2, dv2 = att.attention_backward(do, q, k, v, o, lse, want_dq=False, **how)
    assert none is None and torch.equal(dk, dk2) and torch.equal(dv, dv2)
    if documents_of == 1:
        far = (d + 8) * 2.0 ** -24 * (do.float().abs() * v.float().abs()).sum(-1, keepdim=True) * d ** -0.5
        small = 2.0 ** -25 if dtype == torch.float16 else 0.0  # (half of fp16's smallest step)
        assert (dq.float().abs() <= 2 * far * k.float().abs() + small).all()
        assert (dk.float().abs() <= 2 * (far * q.float().abs()).sum(3, keepdim=True) + small).all()
