"""How the attention half of the particles' layers is called: refusals, streams, graphs, autograd, offsets beyond 32 bits, and together with the other layers and the SVGD step."""
import math
import os
import sys

import pytest
import torch

import attention_reference as ref
from test_gpu_attention import gen, normal, params

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


def block(att, x, batch, tokens, heads, kv, d, weights, frequencies, positions, how):
    """A whole attention block through the autograd functions."""
    w, b, qw, kw, slopes, ow = weights
    n = x.shape[0]
    qkv = att.linear(x, w, b).view(n, batch, tokens, heads + 2 * kv, d)
    q, k = att.qk_norm_rotary(qkv[..., :heads, :], qkv[..., heads:heads + kv, :], qw, kw, frequencies, positions)
    o = att.attention(q, k, qkv[..., heads + kv:, :], slopes=slopes, **how)
    return att.linear(o.flatten(3).view(n, batch * tokens, heads * d), ow, residual=x)


def block_inputs(g, n=2, batch=2, tokens=20, heads=4, kv=2, d=16, dtype=torch.float32, spread=0.3):
    width = heads * d
    x = normal(g, n, batch * tokens, width, dtype=dtype)
    shapes = [((heads + 2 * kv) * d, width), ((heads + 2 * kv) * d,), (d,), (d,), (heads,), (width, width)]
    weights, grads, G, D = params(g, n, 3, *shapes, spread=spread)
    frequencies = torch.tensor([100.0 ** (-2 * j / d) for j in range(d // 2)], dtype=torch.float64, device="cuda")
    return x, weights, grads, G, frequencies, torch.arange(7, 7 + tokens, device="cuda"), (batch, tokens, heads, kv, d)


def test_refusals(att):
    x, w = torch.zeros(2, 3, 8, device="cuda"), torch.zeros(2, 5, 8, device="cuda")
    q, k = torch.zeros(2, 1, 4, 6, 16, device="cuda"), torch.zeros(2, 1, 9, 2, 16, device="cuda")
    o, lse = att.attention_forward(q, k, k)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    f64, pos = torch.ones(4, dtype=torch.float64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    qw = torch.zeros(2, 16, device="cuda")
    k4 = k[:, :, :4]
    cases = [
        (TypeError, "weight must be", lambda: att.linear_forward(x, w.bfloat16())), (TypeError, "particles, out, width", lambda: att.linear_forward(x, w[0])),
        (ValueError, "weight must have the shape", lambda: att.linear_forward(x, w[:1])), (ValueError, "bias must have the shape", lambda: att.linear_forward(x, w, w[:, 0])),
        (ValueError, "activation must be", lambda: att.linear_forward(x, w, activation="swish")), (ValueError, "residual must have the shape", lambda: att.linear_forward(x, w, residual=x)),
        (ValueError, "residual must have the type", lambda: att.linear_forward(x, w, residual=torch.zeros(2, 3, 5, device="cuda").half())),
        (TypeError, "saved must be", lambda: att.linear_backward(torch.zeros(2, 3, 5, device="cuda"), x, w, None, activation="silu")),
        (ValueError, "dy must have the shape", lambda: att.linear_backward(x, x, w)), (att.layers_error, "INVALID_ARG", lambda: att.linear_backward(torch.zeros(2, 3, 5, device="cuda"), x, w, None, w)),
        (TypeError, "q must be", lambda: att.attention_forward(q.double(), k, k)), (TypeError, "q must be", lambda: att.attention_forward(q[0], k, k)),
        (ValueError, "k must have the type", lambda: att.attention_forward(q, k.half(), k)), (ValueError, "v must have the shape", lambda: att.attention_forward(q, k, k4)),
        (ValueError, "multiple", lambda: att.attention_forward(q[..., :5, :], k, k)), (TypeError, "contiguous heads", lambda: att.attention_forward(q.transpose(3, 4), k, k)),
        (TypeError, "lengths must be", lambda: att.attention_forward(q, k, k, lengths=ints(2))), (TypeError, "starts must be", lambda: att.attention_forward(q, k, k, starts=ints(1).long())),
        (TypeError, "documents must be", lambda: att.attention_forward(q, k, k, documents=ints(1, 4))), (TypeError, "prefix must be", lambda: att.attention_forward(q, k, k, prefix=ints(1).cpu())),
        (ValueError, "slopes must have the shape", lambda: att.attention_forward(q, k, k, slopes=torch.zeros(2, 2, device="cuda"))),
        (att.layers_error, "INVALID_ARG", lambda: att.attention_forward(q, k, k, cap=-1.0)), (att.layers_error, "INVALID_ARG", lambda: att.attention_forward(q, k, k, scale=0.0)),
        (att.layers_error, "TOO_LARGE", lambda: att.attention_forward(*[torch.zeros(1, 1, 1, 1, 130, device="cuda")] * 3)),
        (TypeError, "lse must be", lambda: att.attention_backward(o, q, k, k, o, lse[..., :2])), (ValueError, "do must have the shape", lambda: att.attention_backward(k, q, k, k, o, lse)),
        (ValueError, "dslopes need slopes", lambda: att.attention_backward(o, q, k, k, o, lse, dslopes=torch.zeros(2, 6, device="cuda"))),
        (ValueError, "together", lambda: att.qk_norm_rotary_forward(q, k4, qw)), (ValueError, "together", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=f64)),
        (TypeError, "frequencies must be", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=f64.float(), positions=pos)),
        (TypeError, "positions must be", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=f64, positions=pos.int())),
        (ValueError, "positions must have the shape", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=f64, positions=pos[:3])),
        (ValueError, "two values of a head", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=torch.ones(9, dtype=torch.float64, device="cuda"), positions=pos)),
        (ValueError, "layout must be", lambda: att.qk_norm_rotary_forward(q, k4, frequencies=f64, positions=pos, layout="other")), (ValueError, "k must have the shape", lambda: att.qk_norm_rotary_forward(q, k)),
        (ValueError, "need q_weight", lambda: att.qk_norm_rotary_backward(q, k4, q, k4, dq_weight=qw)),
        (att.layers_error, "TOO_LARGE", lambda: att.qk_norm_rotary_forward(*[torch.zeros(1, 1, 1, 1, 258, device="cuda")] * 2)),
    ]
    for error, words, call in cases:
        with pytest.raises(error, match=words):
            call()
            pytest.fail(words)
    torch.cuda.synchronize()


@pytest.fixture(autouse=True)
def _error(att):
    from paper_2306_06528_amd.svgd import SvgdError
    att.layers_error = SvgdError
    yield
    del att.layers_error


def everything(att, x, dy, weights, grads, frequencies, positions, sizes, stream=None):
    """Plain calls of all three, forward and backward."""
    batch, tokens, heads, kv, d = sizes
    w, b, qw, kw, slopes, ow = weights
    dw, db, dqw, dkw, ds, dow = grads
    n = x.shape[0]
    qkv, _ = att.linear_forward(x, w, b, stream=stream)
    qkv = qkv.view(n, batch, tokens, heads + 2 * kv, d)
    q0, k0, v = qkv[..., :heads, :], qkv[..., heads:heads + kv, :], qkv[..., heads + kv:, :]
    rot = {"frequencies": frequencies, "positions": positions, "stream": stream}
    q, k = att.qk_norm_rotary_forward(q0, k0, qw, kw, **rot)
    how = {"causal": True, "cap": 20.0, "slopes": slopes, "stream": stream}
    o, lse = att.attention_forward(q, k, v, **how)
    y, saved = att.linear_forward(o.view(n, batch * tokens, heads * d), ow, None, "gelu", x, save=True, stream=stream)
    do = att.linear_backward(dy, o.view(n, batch * tokens, heads * d), ow, saved, dow, None, "gelu", stream=stream)
    dq, dk, dv = att.attention_backward(do.view(o.shape), q, k, v, o, lse, dslopes=ds, **how)
    dq, dk = att.qk_norm_rotary_backward(dq, dk, q0, k0, qw, kw, dqw, dkw, **rot)
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        dqkv = torch.cat([dq, dk, dv], 3).view(n, batch * tokens, -1)
    return y, att.linear_backward(dqkv, x, w, None, dw, db, stream=stream)


def test_another_stream(att):
    """Calls on a stream that is not the current one wait for what that stream has to do first."""
    g = gen(20)
    x, weights, grads, G, f, p, sizes = block_inputs(g)
    dy = normal(g, *x.shape, dtype=torch.float32)
    want = [t.clone() for t in (*everything(att, x, dy, weights, grads, f, p, sizes), G)]
    side, late = torch.cuda.Stream(), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.randn(1 << 22, device="cuda").sort()
        late.copy_(x)
        G.fill_(-7.0)
    got = everything(att, late, dy, weights, grads, f, p, sizes, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, G), want))


@pytest.mark.parametrize("tokens", [20, 1])
def test_captured_and_replayed(att, tokens):
    """Forward and backward of all of them in one graph, replayed on new inputs between eager work: every replay as the eager call; and a second graph of the same calls."""
    g = gen(21)
    x, weights, grads, G, f, p, sizes = block_inputs(g, tokens=tokens, batch=3)
    dy = normal(g, *x.shape, dtype=torch.float32)
    everything(att, x, dy, weights, grads, f, p, sizes)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(everything(att, x, dy, weights, grads, f, p, sizes))
    for k in range(4):
        x.copy_(torch.randn(x.shape, generator=g).cuda())
        p.add_(k)
        want = [t.clone() for t in (*everything(att, x, dy, weights, grads, f, p, sizes), G)]
        torch.cuda.synchronize()
        for graph, out in zip(graphs, outs):
            for t in grads:
                t.fill_(-3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((*out, G), want)), k


def test_the_same_inputs_give_the_same_bits(att):
    g = gen(22)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        x, weights, grads, G, f, p, sizes = block_inputs(g, tokens=150, dtype=dtype)
        dy = normal(g, *x.shape, dtype=dtype)
        first = [t.clone() for t in (*everything(att, x, dy, weights, grads, f, p, sizes), G)]
        for _ in range(3):
            G[:, 3:-3].fill_(0.0)
            assert all(torch.equal(a, b) for a, b in zip((*everything(att, x, dy, weights, grads, f, p, sizes), G), first))


def test_cache_of_long_strides(att):
    """A cache whose last keys lie beyond 2^31 elements, of which few are filled; and token strides that attention's kernels do not reach, which are copied."""
    g = gen(23)
    big = torch.zeros(1, 2, 9_000, 2, 64_000, dtype=torch.float16, device="cuda")  # 2.3e9 values
    k, v = big[..., 63_000:63_064], big[..., 10_000:10_064]
    k.copy_(normal(g, 1, 2, 9_000, 2, 64, dtype=torch.float16))
    v.copy_(normal(g, 1, 2, 9_000, 2, 64, dtype=torch.float16))
    q = normal(g, 1, 2, 1, 4, 64, dtype=torch.float16)
    lengths = torch.tensor([9_000, 8_001], dtype=torch.int32, device="cuda")
    o, lse = att.attention_forward(q, k, v, lengths=lengths)
    want = ref.attention(q, k, v, lengths=lengths)
    ref.check(o, want["o"], "o")
    ref.check_lse(lse, want["lse"])
    far = big.view(-1)[:40 * (1 << 23)].view(1, 1, 40, 1, 1 << 23)[..., :32]
    far.copy_(normal(g, 1, 1, 40, 1, 32, dtype=torch.float16))
    near = far.contiguous()
    o, lse = att.attention_forward(far, far, far, causal=True)
    assert torch.equal(o, att.attention_forward(near, near, near, causal=True)[0])
    for a, b in zip(att.attention_backward(far, far, far, far, o, lse, causal=True), att.attention_backward(near, near, near, near, o, lse, causal=True)):
        assert torch.equal(a, b)


def test_many_heads_of_gradients_beyond_32_bits(att):
    """Rows of one linear map's results further apart than 2^31 elements from first to last."""
    n, batch, t, h, d = 1, 1, 40_000, 1, 64
    wide = torch.empty(n, batch, t, h, 60_000, dtype=torch.bfloat16, device="cuda")  # 2.4e9 values
    g = gen(24)
    q, k = wide[..., 100:100 + d], wide[..., 50_000:50_000 + d]
    q.copy_(torch.randn(q.shape, generator=g).cuda())
    k.copy_(torch.randn(k.shape, generator=g).cuda())
    frequencies, positions = torch.tensor([0.5, 0.25], dtype=torch.float64, device="cuda"), torch.arange(t, device="cuda")
    a, b = att.qk_norm_rotary_forward(q, k, frequencies=frequencies, positions=positions)
    for got, x in ((a, q), (b, k)):
        ref.check(got[:, :, -50:], ref.qk_norm_rotary(x[:, :, -50:], None, frequencies, positions[-50:], "half", 0.0)["y"], "turned")


def test_autograd_matches_the_plain_calls(att):
    g = gen(25)
    x, weights, grads, G, f, p, sizes = block_inputs(g, dtype=torch.bfloat16)
    batch, tokens, heads, kv, d = sizes
    n = x.shape[0]
    dy = normal(g, *x.shape, dtype=torch.bfloat16)
    w, b, qw, kw, slopes, ow = weights
    leaves = [t.detach().requires_grad_() for t in (x, *weights)]
    for t, into in zip(leaves[1:], grads):  # gradients land in G
        into.fill_(0.0)
        t.grad = into
    out = block(att, leaves[0], *sizes, leaves[1:], f, p, {"causal": True, "cap": 20.0})
    out.backward(dy)
    auto = G.clone()
    qkv = att.linear_forward(x, w, b)[0].view(n, batch, tokens, heads + 2 * kv, d)
    q0, k0, v = qkv[..., :heads, :], qkv[..., heads:heads + kv, :], qkv[..., heads + kv:, :]
    q, k = att.qk_norm_rotary_forward(q0, k0, qw, kw, f, p)
    o, lse = att.attention_forward(q, k, v, True, 20.0, slopes)
    flat = o.view(n, batch * tokens, heads * d)
    assert torch.equal(out, att.linear_forward(flat, ow, residual=x)[0])
    do = att.linear_backward(dy, flat, ow, None, grads[5])
    dq, dk, dv = att.attention_backward(do.view(o.shape), q, k, v, o, lse, True, 20.0, slopes, dslopes=grads[4])
    dq, dk = att.qk_norm_rotary_backward(dq, dk, q0, k0, qw, kw, grads[2], grads[3], f, p)
    dx = att.linear_backward(torch.cat([dq, dk, dv], 3).view(n, batch * tokens, -1), x, w, None, grads[0], grads[1])
    assert torch.equal(auto, G) and torch.equal(leaves[0].grad, dx + dy)


def test_autograd_of_shared_inputs_and_sums(att):
    """A batch that all particles share gets the sum of their gradients; a sum's gradient has no strides; only some gradients wanted."""
    g = gen(26)
    x, weights, _, _, f, p, sizes = block_inputs(g, n=3)
    shared = x[0].clone().requires_grad_()
    block(att, shared.expand(3, -1, -1), *sizes, weights, f, p, {"causal": True}).sum().backward()
    each = x[:1].expand(3, -1, -1).clone().requires_grad_()
    block(att, each, *sizes, weights, f, p, {"causal": True}).sum().backward()
    # the same values added up in another order
    assert (shared.grad - each.grad.sum(0)).abs().max() <= 4 * ref.U * each.grad.abs().sum(0).max()
    k = normal(g, 1, 1, 30, 2, 16, dtype=torch.float32)
    one = k.clone().requires_grad_()
    att.attention(k.expand(2, -1, -1, -1, -1), one.expand(2, -1, -1, -1, -1), k.expand(2, -1, -1, -1, -1)).sum().backward()
    assert one.grad.shape == k.shape and torch.isfinite(one.grad).all()
    s = weights[4].detach().clone().requires_grad_()
    att.attention(normal(g, 3, 1, 9, 4, 16, dtype=torch.float32), normal(g, 3, 1, 9, 4, 16, dtype=torch.float32), normal(g, 3, 1, 9, 4, 16, dtype=torch.float32), slopes=s).sum().backward()
    assert torch.isfinite(s.grad).all()


@pytest.mark.parametrize("how", [{"causal": True}, {"cap": 3.0}, {"causal": True, "prefix": True}, {"documents": True}])
def test_gradients_against_differences(att, how):
    """The whole block's gradient along a direction against a central difference of its value: both in fp32, differences of 2e-2 of values around 1, a cubic term below 1e-3."""
    g = gen(27)
    x, weights, _, _, f, p, sizes = block_inputs(g, tokens=12)
    how = dict(how)
    if "prefix" in how:
        how["prefix"] = torch.tensor([5, 0], dtype=torch.int32, device="cuda")
    if "documents" in how:
        how["documents"] = torch.tensor([[0] * 5 + [1] * 7, [2] * 12], dtype=torch.int32, device="cuda")
    c = normal(g, *x.shape, dtype=torch.float32).double()
    leaves = [t.detach().clone().requires_grad_() for t in (x, *weights)]

    def value(ts):
        return (block(att, ts[0], *sizes, ts[1:], f, p, how).double() * c).sum()

    value(leaves).backward()
    for k, leaf in enumerate(leaves):
        d = torch.randn(leaf.shape, generator=g).cuda()
        d /= d.norm()
        t = 1e-2
        sides = [value([q.detach() + (s * t * d if i == k else 0) for i, q in enumerate(leaves)]).item() for s in (1, -1)]
        slope = (leaf.grad.double() * d).sum().item()
        size = (leaf.grad.double() ** 2).sum().sqrt().item()
        assert abs((sides[0] - sides[1]) / (2 * t) - slope) <= 2e-3 * size, k


def test_tangents_are_refused(att):
    import torch.autograd.forward_ad as forward_ad
    q, x, w = torch.ones(1, 1, 2, 1, 4, device="cuda"), torch.ones(1, 2, 4, device="cuda"), torch.ones(1, 3, 4, device="cuda")
    for call, t in ((lambda t: att.linear(t, w), x), (lambda t: att.linear(x, t), w), (lambda t: att.qk_norm_rotary(t, q), q), (lambda t: att.attention(q, t, q), q)):
        for mode in (torch.enable_grad, torch.no_grad):
            with forward_ad.dual_level(), mode(), pytest.raises(NotImplementedError):
                call(forward_ad.make_dual(t, torch.ones_like(t)))
                pytest.fail("a tangent was lost")


# ---------------------------------------------------------------------------------------------
# together with the other layers and the SVGD step
# ---------------------------------------------------------------------------------------------
def test_scores_of_the_example():
    """The scores that the example leaves in G are those that autograd finds for the same networks in plain torch, in 64 bits."""
    import attention_blocks
    n, width, batch, tokens = 2, 32, 2, 11
    net = attention_blocks.Ensemble(n, width, 2, seed=3)
    g = gen(28)
    x, c = torch.randn(batch, tokens, width, generator=g).cuda(), torch.randn(n, batch, tokens, generator=g).cuda()
    out = net.forward(x)
    (out * c).sum().backward()
    leaves = [t.detach().double().cpu().clone().requires_grad_() for t in net.leaves]
    s, at, heads, kv, d = x.double().cpu().view(1, batch * tokens, width).expand(n, -1, -1), 0, net.heads, net.kv, net.dim
    angle = (torch.arange(tokens).double()[:, None] * net.frequencies.cpu())[None, :, None]
    far = (torch.arange(tokens)[:, None] - torch.arange(tokens)).double()

    def norm(s, w, b):
        m = s - s.mean(-1, keepdim=True)
        return m * (m.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w[:, None] + b[:, None]

    for _ in net.blocks:
        n1, b1, qkv, qb, qn, kn, sl, ow, n2, b2, gate, up, down = leaves[at:at + 13]
        at += 13
        z = (norm(s, n1, b1) @ qkv.transpose(1, 2) + qb[:, None]).view(n, batch, tokens, heads + 2 * kv, d)
        qk = []
        for part, w in ((z[..., :heads, :], qn), (z[..., heads:heads + kv, :], kn)):
            part = part * (part.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w[:, None, None, None]
            a, b = part.chunk(2, -1)
            qk.append(torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).transpose(2, 3))
        k, v = (t.repeat_interleave(heads // kv, 2) for t in (qk[1], z[..., heads + kv:, :].transpose(2, 3)))
        score = qk[0] @ k.transpose(-1, -2) * d ** -0.5 - sl[:, None, :, None, None] * far.abs()
        o = torch.softmax(score.masked_fill(far < 0, -math.inf), -1) @ v
        s = s + o.transpose(2, 3).reshape(n, batch * tokens, heads * d) @ ow.transpose(1, 2)
        h = norm(s, n2, b2)
        s = s + (torch.nn.functional.silu(h @ gate.transpose(1, 2)) * (h @ up.transpose(1, 2))) @ down.transpose(1, 2)
    want = (s @ leaves[at].transpose(1, 2)).view(n, batch, tokens)
    (want * c.double().cpu()).sum().backward()
    # two blocks of fp32 products over up to 96 values: some hundred roundings of 2^-24 of the largest terms
    assert (out.detach().double().cpu() - want).abs().max() <= 2e-5 * want.abs().max()
    G = torch.cat([t.grad.reshape(n, -1) for t in leaves], 1)
    assert G.shape == net.G.shape and (net.G.double().cpu() - G).abs().max() <= 2e-5 * G.abs().max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_example_runs_and_continues_token_by_token(dtype):
    import attention_blocks
    net, x, y, history = attention_blocks.train(n=4, width=32, batch=3, tokens=20, steps=5, dtype=dtype, report=lambda line: None)
    assert torch.isfinite(history).all() and torch.isfinite(net.X).all()
    with torch.no_grad():
        whole = net.forward(x)
    parts = net.continued(x, 8)
    # fp32: another order of sums; bf16: each of some ten activations on the way is rounded once, by half a step of 2^-8 of it, and values of that size are added up with other signs
    assert (whole.float() - parts.float()).abs().max() <= (1e-4 if dtype == torch.float32 else 12 * 2.0 ** -8) * whole.float().abs().max()
