"""Queries that see nothing, whatever they and the gradient of their o hold: o and dq are 0, and nothing of them is in dk, dv and the slopes' gradients.  So it is with a batch that is padded on the left
(queries before the first key), and with empty sequences."""
import math

import pytest
import torch

import attention_reference as ref
from test_gpu_attention import IDS, TYPES, gen, normal, params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


CASES = {  # batch, tokens, keys, how
    "left_padded": (3, 100, 100, lambda: {"causal": True, "starts": ints(-30, 0, -99)}),
    "left_padded_cache": (3, 7, 300, lambda: {"causal": True, "starts": ints(-3, 290, -7), "lengths": ints(4, 297, 0)}),
    "empty": (4, 70, 90, lambda: {"lengths": ints(0, 90, 33, 0)}),
    "more_queries_than_keys": (2, 150, 80, lambda: {"causal": True}),
    "documents": (2, 90, 90, lambda: {"documents": (torch.arange(90, dtype=torch.int32)[None].expand(2, -1) // 20).contiguous().cuda(), "starts": ints(-25, 30)}),
    "in_parts": (1, 1_700, 1_600, lambda: {"causal": True, "starts": ints(-200)}),
}


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv,d,biased", [(4, 2, 40, True), (2, 2, 64, False), (6, 2, 128, False)])
@pytest.mark.parametrize("name", CASES)
def test_nothing_flows_back(att, name, heads, kv, d, biased, dtype):
    batch, t, s, how = CASES[name]
    how, g, n = how(), gen(name, d), 2 if name != "in_parts" else 1
    q, do = (normal(g, n, batch, t, heads, d, dtype=dtype) for _ in range(2))
    k, v = (normal(g, n, batch, s, kv, d, dtype=dtype) for _ in range(2))
    ds = None
    if biased:
        (how["slopes"],), (ds,), G, _ = params(g, n, 2, (heads,), spread=0.05)
    see, _ = ref.seen(batch, t, s, **{x: m for x, m in how.items() if x != "slopes"})
    blind = (~see.any(-1)).cuda()
    assert blind.any() and not blind.all()
    hidden = blind[None, :, :, None, None]
    q, do = (torch.where(hidden, torch.zeros((), dtype=dtype, device="cuda"), x) for x in (q, do))
    want = ref.attention(q, k, v, do, **how)
    for bad in (math.nan, math.inf):
        x, dx = (torch.where(hidden, torch.full((), bad, dtype=dtype, device="cuda"), y) for y in (q, do))
        o, lse = att.attention_forward(x, k, v, **how)
        got = dict(zip(("o", "dq", "dk", "dv"), (o, *att.attention_backward(dx, x, k, v, o, lse, dslopes=ds, **how))))
        if biased:
            got["dslopes"] = ds
        ref.check_lse(lse, want["lse"])
        for key, y in got.items():
            ref.check(y, want[key], f"{key} with {bad}")
        assert (o[:, blind] == 0).all() and (got["dq"][:, blind] == 0).all()
        _, dk, dv = att.attention_backward(dx, x, k, v, o, lse, want_dq=False, **how)
        ref.check(dk, want["dk"], "dk alone")  # (fp32's delta is then a sum in another order: within (d + 8) U of its terms, which the bound has)
        assert torch.equal(dv, got["dv"])
