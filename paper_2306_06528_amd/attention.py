"""The attention half of the particles' layers on all n networks at once: linear maps with bias, activation and residual, norms of queries
and keys with the rotation by their positions, and attention, forward and backward (include/svgd_attention.h, in the same libsvgd.so;
here and in csrc/attention_binding.cpp arguments are checked and handed on).  What layers.py says holds here too: activations are CUDA
tensors of float32, bfloat16 or float16, parameters float32 views into the rows of X, their gradients views of the same places of G,

    weight, dweight = (M[:, a:a + f * d].view(n, f, d) for M in (X, G))         # linear: (n, out, width)
    bias, dbias = X[:, b:b + f], G[:, b:b + f]                                  # (n, out)
    q_weight, dq_weight = X[:, c:c + dim], G[:, c:c + dim]                      # norms: (n, dim)
    slopes, dslopes = X[:, s:s + heads], G[:, s:s + heads]                      # attention: (n, heads)

there are plain calls (`*_forward` / `*_backward`), which can be captured into graphs, and autograd functions (`linear`,
`qk_norm_rotary`, `attention`), and none of them knows forward-mode differentiation.

Activations with heads are (n, batch, tokens, heads, dim); a head's values have to be contiguous, other strides are free: q, k and v may be
views into the results of one linear map,

    qkv = attention.linear(x, weight, bias).view(n, batch, tokens, heads + 2 * kv_heads, dim)
    q, k, v = qkv[..., :heads, :], qkv[..., heads:heads + kv_heads, :], qkv[..., heads + kv_heads:, :]
    q, k = attention.qk_norm_rotary(q, k, q_weight, k_weight, frequencies, positions)
    s = attention.linear(attention.attention(q, k, v, causal=True).flatten(3).flatten(1, 2), out_weight, residual=s)
"""
import torch

from . import _binding
from .layers import _call, _new_grad, _no_derivatives, _with_rows


# ---------------------------------------------------------------------------------------------
# linear map
# ---------------------------------------------------------------------------------------------
def linear_forward(x, weight, bias=None, activation: str = "none", residual=None, save: bool = False, stream=None):
    """(y, saved): y = act(weight x + bias) + residual row by row; activation "none", "silu", "gelu", "relu" or "tanh".  x is
    (n, ..., width), y and residual are (n, ..., out).  saved, what linear_backward takes, is None without `save` and without an activation."""
    return _call(_binding.linear_forward, stream, x, x, weight, bias, activation, residual, save)


def linear_backward(dy, x, weight, saved=None, dweight=None, dbias=None, activation: str = "none", accumulate: bool = False, want_dx: bool = True,
                    stream=None):
    """dx (or None).  The gradients of weight and bias are written, or with `accumulate` added, to dweight and dbias; where these are None
    they are not wanted.  The residual's gradient is dy."""
    return _call(_binding.linear_backward, stream, x, dy, x, weight, saved, dweight, dbias, activation, accumulate, want_dx)[0]


# ---------------------------------------------------------------------------------------------
# norms of queries and keys, rotation
# ---------------------------------------------------------------------------------------------
def qk_norm_rotary_forward(q, k, q_weight=None, k_weight=None, frequencies=None, positions=None, layout: str = "half", eps: float = 1e-6, stream=None):
    """(q, k): every head divided by its root mean square and multiplied by q_weight or k_weight (both None: no norm), then its pairs
    of values j turned by position * frequencies[j] (float64, angle per token): the values j and j + len(frequencies) with layout "half", 2 j and 2 j + 1 with
    "interleaved".  What lies behind the pairs stays.  positions: int64, (tokens,) or (batch, tokens).  frequencies and positions None: no rotation."""
    return _call(_binding.qk_norm_rotary_forward, stream, q, q, k, q_weight, k_weight, frequencies, positions, layout, eps)


def qk_norm_rotary_backward(dq, dk, q, k, q_weight=None, k_weight=None, dq_weight=None, dk_weight=None, frequencies=None, positions=None,
                            layout: str = "half", eps: float = 1e-6, accumulate: bool = False, stream=None):
    """(dq, dk): the gradients of the q and k that the forward call took, from those of its results.  The weights' gradients are written, or
    with `accumulate` added, to dq_weight and dk_weight; where one is None it is not wanted."""
    return _call(_binding.qk_norm_rotary_backward, stream, q, dq, dk, q, k, q_weight, k_weight, frequencies, positions, layout, eps, dq_weight, dk_weight,
                 accumulate)


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------
def attention_forward(q, k, v, causal: bool = False, cap: float = 0.0, slopes=None, scale=None, starts=None, lengths=None, documents=None, prefix=None,
                      stream=None):
    """(o, lse): o = softmax(scores) v, where the score of query i and key j is z = scale q_i k_j (scale None: 1 / sqrt(dim)), capped to
    cap tanh(z / cap) unless cap is 0, less slopes times the distance of their positions if slopes are given, (n, heads).  q is (n, batch, tokens, heads, dim), k and v
    (n, batch, keys, kv_heads, dim), heads a multiple of kv_heads: successive heads share a key head.

    Key j is at position j, query i at starts[b] + i (None: the queries are the last tokens, keys - tokens + i).  All masks are int32 CUDA tensors: with `causal` a
    query sees no key behind its position, but the first prefix[b] in any case; lengths (batch,): how many keys there are (what lies behind is not read: a cache that was filled so
    far; before that keys and values have to be finite, seen or not); documents (batch, keys): a query sees only keys of its position's document.  A query that sees nothing has o = 0 and lse = -inf,
    and nothing flows back from it.
    lse, float32 (n, batch, heads, tokens), is for attention_backward.  One call serves training, prompts and single tokens over a cache."""
    return _call(_binding.attention_forward, stream, q, q, k, v, causal, cap, slopes, scale, starts, lengths, documents, prefix)


def attention_backward(do, q, k, v, o, lse, causal: bool = False, cap: float = 0.0, slopes=None, scale=None, starts=None, lengths=None, documents=None,
                       prefix=None, dslopes=None, accumulate: bool = False, want_dq: bool = True, want_dkv: bool = True, stream=None):
    """(dq, dk, dv), None where not wanted; o and lse are what attention_forward returned.  The slopes' gradients are written, or with `accumulate` added, to dslopes; None:
    not wanted."""
    return _call(_binding.attention_backward, stream, q, do, q, k, v, o, lse, causal, cap, slopes, scale, starts, lengths, documents, prefix, dslopes,
                 accumulate, want_dq, want_dkv)


# ---------------------------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------------------------
def _with_heads(d):
    """A gradient as autograd hands it over may be expanded (from a sum) or transposed."""
    return d if d.shape[-1] == 1 or d.stride(-1) == 1 else d.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, activation, residual, grad_enabled):
        y, saved = linear_forward(x, weight, bias, activation, residual, save=grad_enabled and any(ctx.needs_input_grad[:3]))
        ctx.save_for_backward(x, weight, bias, saved)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, saved = ctx.saved_tensors
        want_dx, want_dw, want_db, _, want_dr, _ = ctx.needs_input_grad
        dx = dw = db = None
        if want_dx or want_dw or want_db:
            dw, db = _new_grad(want_dw, weight), _new_grad(want_db, bias)
            dx = linear_backward(_with_rows(dy), x, weight, saved, dw, db, ctx.activation, want_dx=want_dx)
        return dx, dw, db, None, dy if want_dr else None, None


class _QkNormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, frequencies, positions, layout, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, frequencies, positions)
        ctx.how = layout, eps
        return qk_norm_rotary_forward(q, k, q_weight, k_weight, frequencies, positions, layout, eps)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        q, k, q_weight, k_weight, frequencies, positions = ctx.saved_tensors
        want_q, want_k, want_qw, want_kw = ctx.needs_input_grad[:4]
        dqw, dkw = _new_grad(want_qw, q_weight), _new_grad(want_kw, k_weight)
        dq, dk = qk_norm_rotary_backward(_with_heads(dq), _with_heads(dk), q, k, q_weight, k_weight, dqw, dkw, frequencies, positions, *ctx.how)
        return dq if want_q else None, dk if want_k else None, dqw, dkw, None, None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, causal, cap, scale, starts, lengths, documents, prefix):
        o, lse = attention_forward(q, k, v, causal, cap, slopes, scale, starts, lengths, documents, prefix)
        ctx.save_for_backward(q, k, v, o, lse, slopes, starts, lengths, documents, prefix)
        ctx.how = causal, cap, scale
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, slopes, *masks = ctx.saved_tensors
        causal, cap, scale = ctx.how
        want_q, want_k, want_v, want_s = ctx.needs_input_grad[:4]
        ds = _new_grad(want_s, slopes)
        dq, dk, dv = attention_backward(_with_heads(do), q, k, v, o, lse, causal, cap, slopes, scale, *masks, dslopes=ds, want_dq=want_q,
                                        want_dkv=want_k or want_v)
        return dq, dk if want_k else None, dv if want_v else None, ds, *[None] * 7


def linear(x, weight, bias=None, activation: str = "none", residual=None):
    """The linear map as an autograd function of x, weight, bias and residual."""
    if _no_derivatives():
        return linear_forward(x, weight, bias, activation, residual)[0]
    return _Linear.apply(x, weight, bias, activation, residual, torch.is_grad_enabled())


def qk_norm_rotary(q, k, q_weight=None, k_weight=None, frequencies=None, positions=None, layout: str = "half", eps: float = 1e-6):
    """Norms and rotation as an autograd function of q, k and the weights.  Frequencies have no gradient: ones that ask for it are refused."""
    if _no_derivatives():
        return qk_norm_rotary_forward(q, k, q_weight, k_weight, frequencies, positions, layout, eps)
    if isinstance(frequencies, torch.Tensor) and frequencies.requires_grad and torch.is_grad_enabled():
        raise ValueError("frequencies have no gradient: detach them")
    return _QkNormRotary.apply(q, k, q_weight, k_weight, frequencies, positions, layout, eps)


def attention(q, k, v, causal: bool = False, cap: float = 0.0, slopes=None, scale=None, starts=None, lengths=None, documents=None, prefix=None):
    """Attention as an autograd function of q, k, v and slopes."""
    if _no_derivatives():
        return attention_forward(q, k, v, causal, cap, slopes, scale, starts, lengths, documents, prefix)[0]
    return _Attention.apply(q, k, v, slopes, causal, cap, scale, starts, lengths, documents, prefix)
