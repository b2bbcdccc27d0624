"""The particles' own layers on all n networks at once: layer norm, gated feed-forward block and dropout, forward and
backward (include/svgd_layers.h, in the same libsvgd.so; argument marshalling only, as in svgd.py).

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

Everything runs on `stream` (a torch stream of the tensors' device), or on the current one; results and scratch memory are
allocated for that stream.  A graph that a user captures around the autograd functions is subject to torch's rules for such captures;
no gradient of these leaves may be pending from an eager pass.
"""
import contextlib
import ctypes

import torch

from . import svgd
from .svgd import SVGD_OK, SvgdError

_lib = svgd._lib


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("particle_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


_int, _i64, _ptr, _size = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
_lib.svgd_layer_norm_forward.argtypes = [_int, _int, _i64, _i64, _Rows, _ptr, _i64, _ptr, _i64, ctypes.c_double, _Rows, _ptr, _ptr, _ptr]
_lib.svgd_layer_norm_scratch.argtypes = [_int, _i64, _i64]
_lib.svgd_layer_norm_backward.argtypes = [_int, _int, _i64, _i64, _Rows, _Rows, _ptr, _i64, _ptr, _ptr, _Rows, _ptr, _i64, _ptr, _i64, _int, _ptr,
                                          _size, _ptr]
_lib.svgd_gated_ffn_buffer.argtypes = [_int, _i64, _i64, _i64, _int]
_lib.svgd_gated_ffn_forward.argtypes = [_int, _int, _int, _i64, _i64, _i64, _Rows, _ptr, _i64, _ptr, _i64, _ptr, _i64, _Rows, _int, _ptr, _size, _ptr]
_lib.svgd_gated_ffn_scratch.argtypes = [_int, _i64, _i64, _i64]
_lib.svgd_gated_ffn_backward.argtypes = [_int, _int, _int, _i64, _i64, _i64, _Rows, _Rows, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _size, _Rows,
                                         _ptr, _i64, _ptr, _i64, _ptr, _i64, _int, _ptr, _size, _ptr]
_lib.svgd_dropout.argtypes = [_int, _int, _i64, _i64, _Rows, _Rows, _Rows, ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64, _ptr, _ptr]
for _f in ("svgd_layer_norm_forward", "svgd_layer_norm_backward", "svgd_gated_ffn_forward", "svgd_gated_ffn_backward", "svgd_dropout"):
    getattr(_lib, _f).restype = _int
for _f in ("svgd_layer_norm_scratch", "svgd_gated_ffn_buffer", "svgd_gated_ffn_scratch"):
    getattr(_lib, _f).restype = _size

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACTIVATIONS = {"silu": 0, "gelu": 1}
_NONE = _Rows(None, 0, 0)


def _check(rc):
    if rc != SVGD_OK:
        raise SvgdError(rc)


def _act(t, name, like=None):
    """An activation as (n, rows, width), checked; `like`: of that one's shape, type and device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in _DTYPES or t.dim() < 2:
        raise TypeError(f"{name} must be a CUDA tensor (particles, ..., width) of float32, bfloat16 or float16")
    if like is not None and (t.shape != like.shape or t.dtype is not like.dtype or t.device != like.device):
        raise ValueError(f"{name} must have the shape, type and device of the other activations")
    if t.dim() == 2:
        t = t.unsqueeze(1)
    elif t.dim() > 3:
        t = t.reshape(t.shape[0], -1, t.shape[-1]) if t.numel() else t.new_empty(t.shape[0], t.shape[1:-1].numel(), t.shape[-1])
    if t.shape[2] != 1 and t.stride(2) != 1 and t.numel():
        raise TypeError(f"{name} must have contiguous rows")
    return t


def _rows(t):
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _param(t, name, shape, device):
    """A parameter or its gradient: float32, the particles' parts contiguous; returns (pointer, stride)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not torch.float32:
        raise TypeError(f"{name} must be a float32 CUDA tensor")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have the shape {shape}, not {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on the device of the activations")
    size = 1
    for d in reversed(range(1, t.dim())):
        if t.shape[d] != 1 and t.stride(d) != size:
            raise TypeError(f"{name} must be contiguous within each particle")
        size *= t.shape[d]
    return t.data_ptr(), (t.stride(0) if shape[0] != 1 else size)


def _grad(t, name, shape, device):
    return (None, 0) if t is None else _param(t, name, shape, device)


@contextlib.contextmanager
def _on(device, stream):
    """The device and stream that a call runs and allocates on; yields the stream as a pointer."""
    if stream is not None and stream.device != device:
        raise ValueError("the stream must be of the activations' device")
    with torch.cuda.stream(stream) if stream is not None else torch.cuda.device(device):
        yield svgd._stream_ptr(None)


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------
def layer_norm_forward(x, weight, bias=None, eps: float = 1e-5, stream=None):
    """(y, mean, rstd): y = (x - mean) rstd weight + bias row by row, weight and bias (n, width).  mean and rstd (float32,
    one per row) are for layer_norm_backward."""
    x3 = _act(x, "x")
    n, rows, width = x3.shape
    w, ws = _param(weight, "weight", (n, width), x.device)
    b, bs = _grad(bias, "bias", (n, width), x.device)
    with _on(x.device, stream) as sp:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean, rstd = torch.empty(2, *x.shape[:-1], dtype=torch.float32, device=x.device)
        _check(_lib.svgd_layer_norm_forward(_DTYPES[x.dtype], n, rows, width, _rows(x3), w, ws, b, bs, float(eps),
                                            _Rows(y.data_ptr(), rows * width, width), mean.data_ptr(), rstd.data_ptr(), sp))
    return y, mean, rstd


def _stats(t, name, x):
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != x.shape[:-1] or t.device != x.device or not t.is_contiguous():
        raise TypeError(f"{name} must be what layer_norm_forward returned for x")
    return t.data_ptr()


def layer_norm_backward(dy, x, weight, mean, rstd, dweight=None, dbias=None, accumulate: bool = False, want_dx: bool = True, stream=None):
    """dx (or None).  The gradients of weight and bias are written, or with `accumulate` added, to dweight and dbias, (n, width) views
    into G for example; where these are None they are not wanted."""
    x3 = _act(x, "x")
    dy3 = _act(dy, "dy", x)
    n, rows, width = x3.shape
    w, ws = _param(weight, "weight", (n, width), x.device)
    gw, gws = _grad(dweight, "dweight", (n, width), x.device)
    gb, gbs = _grad(dbias, "dbias", (n, width), x.device)
    m, r = _stats(mean, "mean", x), _stats(rstd, "rstd", x)
    with _on(x.device, stream) as sp:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_dx else None
        nbytes = _lib.svgd_layer_norm_scratch(n, rows, width) if gw or gb else 0
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
        _check(_lib.svgd_layer_norm_backward(_DTYPES[x.dtype], n, rows, width, _rows(dy3), _rows(x3), w, ws, m, r,
                                             _Rows(dx.data_ptr(), rows * width, width) if want_dx else _NONE, gw, gws, gb, gbs, int(bool(accumulate)),
                                             scratch.data_ptr() if nbytes else None, nbytes, sp))
    return dx


# ---------------------------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------------------------
def _block(x3, gate, up, down, activation):
    n, rows, width = x3.shape
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {tuple(_ACTIVATIONS)}")
    if not isinstance(gate, torch.Tensor) or gate.dim() != 3:
        raise TypeError("gate must be a float32 CUDA tensor (particles, hidden, width)")
    hidden = gate.shape[1]
    params = (*_param(gate, "gate", (n, hidden, width), x3.device), *_param(up, "up", (n, hidden, width), x3.device),
              *_param(down, "down", (n, width, hidden), x3.device))
    return (_ACTIVATIONS[activation], n, rows, width, hidden), params


def gated_ffn_forward(x, gate, up, down, activation: str = "silu", save: bool = False, stream=None):
    """(y, saved): y = down (act(gate x) * (up x)) row by row.  saved, what gated_ffn_backward takes, is None without `save`."""
    x3 = _act(x, "x")
    sizes, params = _block(x3, gate, up, down, activation)
    _, n, rows, width, hidden = sizes
    with _on(x.device, stream) as sp:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        nbytes = _lib.svgd_gated_ffn_buffer(n, rows, width, hidden, int(bool(save)))
        buffer = torch.empty(nbytes // 4, dtype=torch.float32, device=x.device)
        _check(_lib.svgd_gated_ffn_forward(_DTYPES[x.dtype], *sizes, _rows(x3), *params, _Rows(y.data_ptr(), rows * width, width), int(bool(save)),
                                           buffer.data_ptr(), nbytes, sp))
    return y, (buffer if save else None)


def gated_ffn_backward(dy, x, gate, up, down, saved, dgate=None, dup=None, ddown=None, activation: str = "silu", accumulate: bool = False,
                       want_dx: bool = True, stream=None):
    """dx (or None).  The gradients of the parameters are written, or with `accumulate` added, to dgate, dup and ddown, which have the
    parameters' shapes; where one is None it is not wanted."""
    x3 = _act(x, "x")
    dy3 = _act(dy, "dy", x)
    sizes, params = _block(x3, gate, up, down, activation)
    _, n, rows, width, hidden = sizes
    grads = (*_grad(dgate, "dgate", (n, hidden, width), x.device), *_grad(dup, "dup", (n, hidden, width), x.device),
             *_grad(ddown, "ddown", (n, width, hidden), x.device))
    need = _lib.svgd_gated_ffn_buffer(n, rows, width, hidden, 1)
    if (not isinstance(saved, torch.Tensor) or saved.dtype is not torch.float32 or saved.numel() * 4 != need or saved.device != x.device
            or not saved.is_contiguous()):
        raise TypeError("saved must be what gated_ffn_forward returned for x with save=True")
    with _on(x.device, stream) as sp:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_dx else None
        nbytes = _lib.svgd_gated_ffn_scratch(n, rows, width, hidden)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        _check(_lib.svgd_gated_ffn_backward(_DTYPES[x.dtype], *sizes, _rows(dy3), _rows(x3), *params, saved.data_ptr(), need,
                                            _Rows(dx.data_ptr(), rows * width, width) if want_dx else _NONE, *grads, int(bool(accumulate)),
                                            scratch.data_ptr(), nbytes, sp))
    return dx


# ---------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------
def dropout_forward(x, p: float, seed: int, call: int = 0, residual=None, counter=None, stream=None):
    """x with every value dropped with probability p, the others divided by 1 - p, plus `residual` if given.  Which values are
    dropped is a function of (seed, call, index): `call` tells the layers and steps of a program apart.  `counter`, an int64 CUDA
    tensor of one element, is read when the kernel runs and changes them too: a replayed graph draws anew where the program counts it
    on."""
    x3 = _act(x, "x")
    res = _act(residual, "residual", x) if residual is not None else None
    n, rows, width = x3.shape
    if counter is not None and (not isinstance(counter, torch.Tensor) or counter.dtype is not torch.int64 or counter.numel() != 1
                                or counter.device != x.device):
        raise TypeError("counter must be an int64 tensor of one element on the device of x")
    with _on(x.device, stream) as sp:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _check(_lib.svgd_dropout(_DTYPES[x.dtype], n, rows, width, _rows(x3), _rows(res) if res is not None else _NONE,
                                 _Rows(y.data_ptr(), rows * width, width), float(p), int(seed) & (2 ** 64 - 1), int(call) & (2 ** 64 - 1),
                                 counter.data_ptr() if counter is not None else None, sp))
    return y


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
    def forward(ctx, x, gate, up, down, activation):
        y, saved = gated_ffn_forward(x, gate, up, down, activation, save=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, gate, up, down, saved)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, gate, up, down, saved = ctx.saved_tensors
        want_dx, *want, _ = ctx.needs_input_grad
        grads = [_new_grad(w, p) for w, p in zip(want, (gate, up, down))]
        dx = gated_ffn_backward(_with_rows(dy), x, gate, up, down, saved, *grads, ctx.activation, want_dx=want_dx)
        return dx, *grads, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, call, residual, counter):
        ctx.draw = (p, seed, call)
        # (the caller moves the counter on between the passes: what this one has drawn with is kept)
        ctx.counter = counter.clone() if counter is not None and ctx.needs_input_grad[0] else None
        return dropout_forward(x, p, seed, call, residual, counter)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = dropout_backward(_with_rows(dy), *ctx.draw, ctx.counter) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dy if ctx.needs_input_grad[4] else None, None


def layer_norm(x, weight, bias=None, eps: float = 1e-5):
    """Layer norm as an autograd function of x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


def gated_ffn(x, gate, up, down, activation: str = "silu"):
    """The gated feed-forward block as an autograd function of x and its three parameters."""
    return _GatedFfn.apply(x, gate, up, down, activation)


def dropout(x, p: float, seed: int, call: int = 0, residual=None, counter=None):
    """Dropout, and the addition to a residual stream, as an autograd function of x and residual."""
    return _Dropout.apply(x, p, seed, call, residual, counter)
