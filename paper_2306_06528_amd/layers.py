"""The particles' own layers on all n networks at once: layer norm, gated feed-forward block and dropout, forward and
backward (include/svgd_layers.h, in the same libsvgd.so; here and in csrc/layers_binding.cpp arguments are checked and handed on).

Activations are CUDA tensors (n, ..., width) of float32, bfloat16 or float16: particle i's rows are t[i].  Rows have to
be contiguous (stride 1 in the last dimension); (n, rows, width) may have any other strides, an expanded batch among them
(`batch.expand(n, -1, -1)`: every particle sees the same rows); more dimensions than three are viewed as three, and copied
where that is not possible.

Parameters are float32 with one leading dimension for the particles, views into the rows of the (n, D) matrix X that
svgd_step moves, and their gradients views of the same places of G:

    weight, dweight = X[:, a:a + d], G[:, a:a + d]                              # layer norm: (n, width)
    gate, dgate = (M[:, b:b + f * d].view(n, f, d) for M in (X, G))             # gate, up: (n, hidden, width)
    down, ddown = (M[:, c:c + d * f].view(n, d, f) for M in (X, G))             # down: (n, width, hidden)

Two ways to use them:

  * `*_forward` / `*_backward`: plain calls.  The gradients of parameters go where the caller says, mostly straight into G
    (`accumulate=True` adds them to what is there); these can be captured into graphs.
  * `layer_norm`, `gated_ffn`, `dropout`: the same as autograd functions, for networks that autograd differentiates.
    Parameters are leaves (`X[:, a:b].detach().requires_grad_()`) whose .grad is a view into G, or any other
    tensors.

Neither knows forward-mode differentiation: the autograd functions refuse a tensor with a tangent, the plain calls do not look for one.

Everything runs on `stream` (a torch stream of the tensors' device), or on the current one; results and scratch memory are
allocated for that stream.  A graph that a user captures around the autograd functions is subject to torch's rules for such captures;
no gradient of these leaves may be pending from an eager pass.
"""
import torch
from torch.autograd import forward_ad

from . import _binding
from .svgd import SvgdError, _cuda_getCurrentRawStream, _cuda_getDevice


def _call(f, stream, x, *args):
    """A call of the native binding (csrc/layers_binding.cpp), which checks the tensors, allocates and calls the library: on the current
    stream of x's device, or on `stream`."""
    if stream is not None:
        if isinstance(x, torch.Tensor) and stream.device != x.device:
            raise ValueError("the stream must be of the activations' device")
        with torch.cuda.stream(stream):
            out = f(_cuda_getDevice, _cuda_getCurrentRawStream, *args)
    else:
        out = f(_cuda_getDevice, _cuda_getCurrentRawStream, *args)
        if out is None:  # x is on another device: nothing has been done
            with torch.cuda.device(x.device):
                out = f(_cuda_getDevice, _cuda_getCurrentRawStream, *args)
    if type(out) is int:
        raise SvgdError(out)
    return out


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------
def layer_norm_forward(x, weight, bias=None, eps: float = 1e-5, stream=None):
    """(y, mean, rstd): y = (x - mean) rstd weight + bias row by row, weight and bias (n, width).  mean and rstd (float32,
    one per row) are for layer_norm_backward."""
    return _call(_binding.layer_norm_forward, stream, x, x, weight, bias, eps)


def layer_norm_backward(dy, x, weight, mean, rstd, dweight=None, dbias=None, accumulate: bool = False, want_dx: bool = True, stream=None):
    """dx (or None).  The gradients of weight and bias are written, or with `accumulate` added, to dweight and dbias, (n, width) views
    into G for example; where these are None they are not wanted."""
    return _call(_binding.layer_norm_backward, stream, x, dy, x, weight, mean, rstd, dweight, dbias, accumulate, want_dx)[0]


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------
def gated_ffn_forward(x, gate, up, down, activation: str = "silu", save: bool = False, stream=None):
    """(y, saved): y = down (act(gate x) * (up x)) row by row.  saved, what gated_ffn_backward takes, is None without `save`."""
    return _call(_binding.gated_ffn_forward, stream, x, x, gate, up, down, activation, save)


def gated_ffn_backward(dy, x, gate, up, down, saved, dgate=None, dup=None, ddown=None, activation: str = "silu", accumulate: bool = False,
                       want_dx: bool = True, stream=None):
    """dx (or None).  The gradients of the parameters are written, or with `accumulate` added, to dgate, dup and ddown, which have the
    parameters' shapes; where one is None it is not wanted."""
    return _call(_binding.gated_ffn_backward, stream, x, dy, x, gate, up, down, saved, dgate, dup, ddown, activation, accumulate, want_dx)[0]


# ---------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------
def dropout_forward(x, p: float, seed: int, call: int = 0, residual=None, counter=None, stream=None):
    """x with every value dropped with probability p, the others divided by 1 - p, plus `residual` if given.  Which values are
    dropped is a function of (seed, call, index): `call` tells the layers and steps of a program apart.  `counter`, an int64 CUDA
    tensor of one element, is read when the kernel runs and changes them too: a replayed graph draws anew where the program counts it
    on."""
    return _call(_binding.dropout, stream, x, x, p, seed, call, residual, counter)[0]


def dropout_backward(dy, p: float, seed: int, call: int = 0, counter=None, stream=None):
    """The gradient of x: dy with the same values dropped and the others divided by 1 - p.  The residual's gradient is dy."""
    return dropout_forward(dy, p, seed, call, None, counter, stream)


# ---------------------------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------------------------
def _with_rows(dy):
    """A gradient as autograd hands it over may be expanded (from a sum) or transposed."""
    return dy if dy.dim() >= 2 and (dy.shape[-1] == 1 or dy.stride(-1) == 1) else dy.contiguous()


def _new_grad(wanted, like):
    return torch.empty(like.shape, dtype=torch.float32, device=like.device) if wanted else None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        want_dx, want_dw, want_db, _ = ctx.needs_input_grad
        dw, db = _new_grad(want_dw, weight), _new_grad(want_db, weight)
        dx = layer_norm_backward(_with_rows(dy), x, weight, mean, rstd, dw, db, want_dx=want_dx)
        return dx, dw, db, None


class _GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, up, down, activation, grad_enabled):
        y, saved = gated_ffn_forward(x, gate, up, down, activation, save=grad_enabled and any(ctx.needs_input_grad))
        ctx.save_for_backward(x, gate, up, down, saved)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, gate, up, down, saved = ctx.saved_tensors
        want_dx, *want, _, _ = ctx.needs_input_grad
        grads = [_new_grad(w, p) for w, p in zip(want, (gate, up, down))]
        dx = gated_ffn_backward(_with_rows(dy), x, gate, up, down, saved, *grads, ctx.activation, want_dx=want_dx)
        return dx, *grads, None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, call, residual, counter, grad_enabled):
        ctx.draw = (p, seed, call)
        # (the caller moves the counter on between the passes: what this one has drawn with is kept)
        ctx.counter = counter.clone() if counter is not None and grad_enabled and ctx.needs_input_grad[0] else None
        return dropout_forward(x, p, seed, call, residual, counter)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = dropout_backward(_with_rows(dy), *ctx.draw, ctx.counter) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dy if ctx.needs_input_grad[4] else None, None, None


def _no_derivatives():
    """Whether no derivative of either mode can be asked for (torch.no_grad leaves forward mode on): the plain calls will do then, which take
    2.5 us less.  Otherwise autograd, which knows the tensors that carry a tangent, refuses them: the layers have no rule for tangents."""
    return not torch.is_grad_enabled() and forward_ad._current_level < 0


# (Within the functions gradients are always off: whether they are on outside, and g, u and h or the counter are to be kept, is handed over.)
def layer_norm(x, weight, bias=None, eps: float = 1e-5):
    """Layer norm as an autograd function of x, weight and bias."""
    if _no_derivatives():
        return layer_norm_forward(x, weight, bias, eps)[0]
    return _LayerNorm.apply(x, weight, bias, eps)


def gated_ffn(x, gate, up, down, activation: str = "silu"):
    """The gated feed-forward block as an autograd function of x and its three parameters."""
    if _no_derivatives():
        return gated_ffn_forward(x, gate, up, down, activation)[0]
    return _GatedFfn.apply(x, gate, up, down, activation, torch.is_grad_enabled())


def dropout(x, p: float, seed: int, call: int = 0, residual=None, counter=None):
    """Dropout, and the addition to a residual stream, as an autograd function of x and residual."""
    if _no_derivatives():
        return dropout_forward(x, p, seed, call, residual, counter)
    return _Dropout.apply(x, p, seed, call, residual, counter, torch.is_grad_enabled())
