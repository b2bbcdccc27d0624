"""The C ABI of the particles' layers without a GPU: exported symbols, plain C, sizes of scratch memory, and that bad
arguments are refused before anything is launched."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import layer_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "svgd_layers.h")
INVALID, TOO_LARGE = -1, -3


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("particle_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class Library:
    """The C ABI as declared in the header."""
    _Rows = Rows

    def __init__(self):
        from paper_2306_06528_amd import svgd
        self._lib = lib = ctypes.CDLL(svgd.LIB_PATH)
        i, l, p, z, d, u = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double, ctypes.c_uint64
        for name, result, args in (
                ("svgd_layer_norm_forward", i, [i, i, l, l, Rows, p, l, p, l, d, Rows, p, p, p]),
                ("svgd_layer_norm_scratch", z, [i, l, l]),
                ("svgd_layer_norm_backward", i, [i, i, l, l, Rows, Rows, p, l, p, p, Rows, p, l, p, l, i, p, z, p]),
                ("svgd_gated_ffn_buffer", z, [i, l, l, l, i]),
                ("svgd_gated_ffn_forward_scratch", z, [i, l, l, l]),
                ("svgd_gated_ffn_forward", i, [i, i, i, l, l, l, Rows, p, l, p, l, p, l, Rows, i, p, z, p, z, p]),
                ("svgd_gated_ffn_scratch", z, [i, l, l, l]),
                ("svgd_gated_ffn_backward", i, [i, i, i, l, l, l, Rows, Rows, p, l, p, l, p, l, p, z, Rows, p, l, p, l, p, l, i, p, z, p]),
                ("svgd_dropout", i, [i, i, l, l, Rows, Rows, Rows, d, u, u, p, p])):
            getattr(lib, name).restype, getattr(lib, name).argtypes = result, args


@pytest.fixture(scope="module")
def layers():
    return Library()


def test_every_declared_symbol_is_exported(layers):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(svgd_[a-z_]+)\s*\(", text)))
    assert len(names) == 9
    for name in names:
        assert hasattr(layers._lib, name), name


@pytest.mark.parametrize("compiler,std,suffix", [("gcc", "-std=c99", ".c"), ("g++", "-std=c++11", ".cpp")])
def test_header_is_plain_c_and_cpp(tmp_path, compiler, std, suffix):
    src = tmp_path / ("use_header" + suffix)
    src.write_text('#include "svgd_layers.h"\nint main(void) { svgd_rows r = {0, 0, 0}; return (int)r.row_stride + SVGD_F32; }\n')
    r = subprocess.run([compiler, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


# Made-up device addresses, far apart: nothing is read on the host, and every call below is refused before a launch.
X, Y, Z, W, V, U, S, B = (k << 32 for k in range(1, 9))


def norm_forward(L, dtype=0, n=2, rows=3, width=4, x=X, xs=(12, 4), w=W, ws=4, b=V, bs=4, eps=1e-5, y=Y, ys=(12, 4), mean=Z, rstd=U):
    return L._lib.svgd_layer_norm_forward(dtype, n, rows, width, L._Rows(x, *xs), w, ws, b, bs, eps, L._Rows(y, *ys), mean, rstd, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(n=0), INVALID), (dict(rows=-1), INVALID), (dict(width=0), INVALID),
    (dict(n=65), TOO_LARGE), (dict(rows=(1 << 30) + 1), TOO_LARGE), (dict(width=16385), TOO_LARGE),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(w=None), INVALID), (dict(x=X + 2), INVALID), (dict(y=Y + 1), INVALID),
    (dict(w=W + 2), INVALID), (dict(b=V + 1), INVALID), (dict(mean=Z + 2), INVALID), (dict(xs=(-12, 4)), INVALID), (dict(xs=(12, 1 << 60)), INVALID), (dict(xs=(12, 1 << 47)), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(eps=-1.0), INVALID),
    (dict(y=X), INVALID), (dict(y=X + 4), INVALID), (dict(y=W), INVALID), (dict(mean=X + 8), INVALID), (dict(rstd=Z), INVALID), (dict(mean=Y), INVALID),
    (dict(ys=(12, 3)), INVALID), (dict(ys=(11, 4)), INVALID), (dict(ys=(0, 4)), INVALID)])
def test_norm_forward_refuses(layers, bad, status):
    assert norm_forward(layers, **bad) == status


def norm_backward(L, dtype=0, n=2, rows=3, width=4, dy=Y, x=X, w=W, ws=4, mean=Z, rstd=Z + 4096, dx=U, dxs=(12, 4), dw=V, dws=8, db=V + 16, dbs=8,
                  scratch=S, nbytes=1 << 20):
    return L._lib.svgd_layer_norm_backward(dtype, n, rows, width, L._Rows(dy, 12, 4), L._Rows(x, 12, 4), w, ws, mean, rstd, L._Rows(dx, *dxs), dw, dws,
                                           db, dbs, 0, scratch, nbytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=7), INVALID), (dict(n=65), TOO_LARGE), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID),
    (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(scratch=None), INVALID), (dict(scratch=S + 8), INVALID), (dict(nbytes=8), INVALID),
    (dict(dw=V + 2), INVALID), (dict(dws=3), INVALID), (dict(db=V + 8), INVALID), (dict(db=V + 28), INVALID), (dict(dw=W), INVALID),
    (dict(dx=Y), INVALID), (dict(dx=X + 4), INVALID), (dict(dxs=(0, 0)), INVALID), (dict(dx=V), INVALID), (dict(scratch=U), INVALID),
    (dict(dw=X), INVALID), (dict(scratch=V), INVALID)])
def test_norm_backward_refuses(layers, bad, status):
    assert norm_backward(layers, **bad) == status


def ffn_forward(L, dtype=0, act=0, n=2, rows=3, width=4, hidden=5, x=X, g=W, u=W + 80, d=W + 160, stride=60, y=Y, ys=(12, 4), save=1, buffer=B,
                nbytes=1 << 20, scratch=S, sbytes=1 << 30):
    return L._lib.svgd_gated_ffn_forward(dtype, act, n, rows, width, hidden, L._Rows(x, 12, 4), g, stride, u, stride, d, stride, L._Rows(y, *ys), save,
                                         buffer, nbytes, scratch, sbytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=3), INVALID), (dict(act=2), INVALID), (dict(act=-1), INVALID), (dict(n=0), INVALID), (dict(n=65), TOO_LARGE), (dict(hidden=0), INVALID),
    (dict(hidden=(1 << 20) + 1), TOO_LARGE), (dict(width=(1 << 20) + 1), TOO_LARGE), (dict(width=0), INVALID), (dict(x=None), INVALID),
    (dict(g=None), INVALID), (dict(u=None), INVALID), (dict(d=None), INVALID), (dict(y=None), INVALID), (dict(buffer=None), INVALID),
    (dict(buffer=B + 4), INVALID), (dict(nbytes=2303), INVALID), (dict(y=X), INVALID), (dict(y=W), INVALID), (dict(buffer=Y), INVALID),
    (dict(buffer=X), INVALID), (dict(g=W + 2), INVALID), (dict(ys=(3, 4)), INVALID)])
def test_ffn_forward_refuses(layers, bad, status):
    assert ffn_forward(layers, **bad) == status


def ffn_backward(L, dtype=0, act=0, n=2, rows=3, width=4, hidden=5, dy=Y, x=X, p=W, dx=U, dg=V, du=V + 80, dd=V + 160, stride=60, saved=B, sbytes=1 << 20,
                 scratch=S, nbytes=1 << 20):
    return L._lib.svgd_gated_ffn_backward(dtype, act, n, rows, width, hidden, L._Rows(dy, 12, 4), L._Rows(x, 12, 4), p, 60, p + 80, 60, p + 160, 60, saved,
                                          sbytes, L._Rows(dx, 12, 4), dg, stride, du, stride, dd, stride, 0, scratch, nbytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=-1), INVALID), (dict(act=5), INVALID), (dict(rows=-1), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(p=2), INVALID),
    (dict(saved=None), INVALID), (dict(sbytes=2303), INVALID), (dict(saved=B + 8), INVALID), (dict(scratch=None), INVALID), (dict(nbytes=1535), INVALID),
    (dict(scratch=S + 4), INVALID), (dict(dg=V + 160), INVALID), (dict(du=V + 76), INVALID), (dict(dd=V + 84), INVALID), (dict(stride=19), INVALID),
    (dict(dd=V + 164), INVALID),  # the end of one particle's meets the start of the next one's
    (dict(dg=W), INVALID), (dict(dx=X), INVALID), (dict(dx=Y + 4), INVALID), (dict(dx=V), INVALID), (dict(scratch=B), INVALID), (dict(dg=X), INVALID),
    (dict(dd=B), INVALID), (dict(scratch=U), INVALID), (dict(dx=B), INVALID), (dict(n=64, rows=1 << 30, hidden=1 << 20), INVALID)])
def test_ffn_backward_refuses(layers, bad, status):
    assert ffn_backward(layers, **bad) == status


def dropout(L, dtype=0, n=2, rows=3, width=4, x=X, xs=(12, 4), r=None, y=Y, ys=(12, 4), p=0.5, counter=None):
    return L._lib.svgd_dropout(dtype, n, rows, width, L._Rows(x, *xs), L._Rows(r, 12, 4), L._Rows(y, *ys), p, 1, 2, counter, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=9), INVALID), (dict(n=0), INVALID), (dict(n=65), TOO_LARGE), (dict(width=0), INVALID), (dict(p=-0.1), INVALID), (dict(p=1.1), INVALID),
    (dict(p=float("nan")), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(y=X + 4), INVALID), (dict(y=X, ys=(4, 8)), INVALID),
    (dict(r=Y + 4), INVALID), (dict(counter=Z + 4), INVALID), (dict(counter=Y + 8), INVALID), (dict(ys=(0, 4)), INVALID), (dict(r=Z + 2), INVALID)])
def test_dropout_refuses(layers, bad, status):
    assert dropout(layers, **bad) == status


def test_no_rows_is_nothing_to_do(layers):
    """(Gradients of parameters, which have something to do then, are tested on the GPU.)"""
    assert norm_forward(layers, rows=0, x=None, y=None) == 0
    assert ffn_forward(layers, rows=0, x=None, y=None, buffer=None) == 0
    assert norm_backward(layers, rows=0, dy=None, x=None, dx=None, dw=None, db=None, scratch=None) == 0
    assert ffn_backward(layers, rows=0, dy=None, x=None, dx=None, dg=None, du=None, dd=None, saved=None, scratch=None) == 0
    assert dropout(layers, rows=0, x=None, y=None) == 0


def test_scratch_sizes(layers):
    lib = layers._lib
    assert lib.svgd_gated_ffn_buffer(2, 3, 4, 33, 0) == 2 * 3 * 64 * 4
    assert lib.svgd_gated_ffn_buffer(2, 3, 4, 33, 1) == 3 * 2 * 3 * 64 * 4
    assert lib.svgd_gated_ffn_buffer(64, 1 << 30, 1, 1 << 20, 1) == 3 * 64 * (1 << 50) * 4
    assert lib.svgd_layer_norm_scratch(1, 0, 8) == 0
    for bad in ((0, 1, 1), (65, 1, 1), (1, -1, 1), (1, 1, 0), (1, 1, 16385)):
        assert lib.svgd_layer_norm_scratch(*bad) == 0
    for bad in ((0, 1, 1, 1), (65, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, 1, 1, (1 << 20) + 1)):
        assert lib.svgd_gated_ffn_buffer(*bad, 1) == 0 and lib.svgd_gated_ffn_scratch(*bad) == 0


def test_python_refuses_what_is_on_no_gpu():
    from paper_2306_06528_amd import layers
    x, w = torch.zeros(2, 3, 4), torch.zeros(2, 4)
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        layers.layer_norm_forward(x, w)
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        layers.dropout_forward(x, 0.5, 1)
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        layers.gated_ffn_forward(x, w, w, w)


def test_generator_is_the_workloads():
    """The reference's bits are the generator's own: splitmix64's published first outputs for state 0, and the uniforms of this
    package's workloads."""
    from paper_2306_06528_amd import workloads
    assert [ref.splitmix64((k * 0x9E3779B97F4A7C15) % 2 ** 64) for k in range(3)] == [0xE220A8397B1DCDAF, 0x6E789E6AA1B965F4, 0x06C45D188009454F]
    assert ref.splitmix64((ref.splitmix64(7) + 3) % 2 ** 64) == workloads.stream_base(7, 3)
    u = workloads.uniform(7, 3, 1000)  # the upper halves of the hashes: the even values
    assert torch.equal(ref.kept(2000, 0.3, 7, 3)[::2], u >= 0.3)
