"""The C ABI of the attention half of the particles' layers without a GPU: exported symbols, plain C, sizes of scratch memory, and that bad arguments are
refused before anything is launched."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "svgd_attention.h")
INVALID, TOO_LARGE = -1, -3
I32, I64, P, Z, D = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double


class Rows(ctypes.Structure):
    _fields_ = [("data", P), ("particle_stride", I64), ("row_stride", I64)]


class Heads(ctypes.Structure):
    _fields_ = [("data", P), ("particle_stride", I64), ("batch_stride", I64), ("token_stride", I64), ("head_stride", I64)]


class Rotary(ctypes.Structure):
    _fields_ = [("n", I32), ("heads", I32), ("kv_heads", I32), ("dim", I32), ("pairs", I32), ("interleaved", I32), ("batch", I64), ("length", I64),
                ("frequencies", P), ("positions", P), ("positions_stride", I64), ("eps", D), ("q_weight", P), ("k_weight", P), ("q_weight_stride", I64),
                ("k_weight_stride", I64)]


class Attention(ctypes.Structure):
    _fields_ = [("n", I32), ("heads", I32), ("kv_heads", I32), ("dim", I32), ("batch", I64), ("length", I64), ("keys", I64), ("causal", I32), ("scale", D), ("cap", D),
                ("slopes", P), ("slopes_stride", I64), ("starts", P), ("lengths", P), ("documents", P), ("prefix", P)]


@pytest.fixture(scope="module")
def lib():
    from paper_2306_06528_amd import svgd
    lib = ctypes.CDLL(svgd.LIB_PATH)
    a, r = ctypes.POINTER(Attention), ctypes.POINTER(Rotary)
    for name, result, args in (
            ("svgd_linear_saved", Z, [I32, I64, I64]), ("svgd_linear_forward_scratch", Z, [I32, I64, I64, I64]), ("svgd_linear_scratch", Z, [I32, I64, I64, I64]),
            ("svgd_linear_forward", I32, [I32, I32, I32, I64, I64, I64, Rows, P, I64, P, I64, Rows, Rows, P, Z, P, Z, P]),
            ("svgd_linear_backward", I32, [I32, I32, I32, I64, I64, I64, Rows, Rows, P, I64, P, Z, Rows, P, I64, P, I64, I32, P, Z, P]),
            ("svgd_qk_norm_rotary_forward", I32, [I32, r, Heads, Heads, Heads, Heads, P]), ("svgd_qk_norm_rotary_scratch", Z, [r]),
            ("svgd_qk_norm_rotary_backward", I32, [I32, r, Heads, Heads, Heads, Heads, Heads, Heads, P, I64, P, I64, I32, P, Z, P]),
            ("svgd_attention_forward_scratch", Z, [a]), ("svgd_attention_forward", I32, [I32, a, Heads, Heads, Heads, Heads, P, P, Z, P]),
            ("svgd_attention_scratch", Z, [a]),
            ("svgd_attention_backward", I32, [I32, a, Heads, Heads, Heads, Heads, Heads, P, Heads, Heads, Heads, P, I64, I32, P, Z, P])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = result, args
    return lib


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(svgd_[a-z_]+)\s*\(", text)))
    assert len(names) == 12
    for name in names:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("compiler,std,suffix", [("gcc", "-std=c99", ".c"), ("g++", "-std=c++11", ".cpp")])
def test_header_is_plain_c_and_cpp(tmp_path, compiler, std, suffix):
    src = tmp_path / ("use_header" + suffix)
    src.write_text('#include "svgd_attention.h"\nint main(void) { svgd_heads h = {0, 0, 0, 0, 0}; return (int)h.head_stride + SVGD_TANH; }\n')
    r = subprocess.run([compiler, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


# Made-up device addresses, far apart: nothing is read on the host, and every call below is refused before a launch.
X, Y, W, V, U, S, B, R, Q, K, O, L, M, N = (k << 32 for k in range(1, 15))


def linear_forward(lib, dtype=0, act=4, n=2, rows=40, width=4, out=6, x=X, xs=(160, 4), w=W, ws=24, b=V, bs=6, res=None, y=Y, ys=(240, 6), z=B, zn=1 << 20, scratch=S, sn=1 << 20):
    return lib.svgd_linear_forward(dtype, act, n, rows, width, out, Rows(x, *xs), w, ws, b, bs, Rows(res, 240, 6), Rows(y, *ys), z, zn, scratch, sn, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID), (dict(n=0), INVALID), (dict(n=65), TOO_LARGE), (dict(rows=-1), INVALID),
    (dict(rows=(1 << 30) + 1), TOO_LARGE), (dict(width=0), INVALID), (dict(width=(1 << 20) + 1), TOO_LARGE), (dict(out=0), INVALID), (dict(out=(1 << 20) + 1), TOO_LARGE),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(w=None), INVALID), (dict(x=X + 2), INVALID), (dict(w=W + 2), INVALID), (dict(b=V + 1), INVALID), (dict(z=B + 8), INVALID),
    (dict(zn=8), INVALID), (dict(xs=(-160, 4)), INVALID), (dict(ys=(240, 5)), INVALID), (dict(ys=(100, 6)), INVALID), (dict(y=X), INVALID), (dict(y=W), INVALID), (dict(y=V), INVALID),
    (dict(z=Y), INVALID), (dict(z=X), INVALID), (dict(res=Y + 4), INVALID), (dict(res=Y), INVALID), (dict(res=R + 1), INVALID), (dict(res=B), INVALID),
    (dict(rows=300, xs=(1 << 20, 2000), ys=(1 << 20, 6), width=2000, scratch=None), INVALID), (dict(rows=300, xs=(1 << 20, 2000), ys=(1 << 20, 6), width=2000, sn=16), INVALID)])
def test_linear_forward_refuses(lib, bad, status):
    assert linear_forward(lib, **bad) == status


def linear_backward(lib, dtype=0, act=0, n=2, rows=40, width=4, out=6, dy=Y, x=X, w=W, ws=24, z=B, zn=1 << 20, dx=U, dxs=(160, 4), dw=V, dws=30, db=V + 96, dbs=30, scratch=S, sn=1 << 20):
    return lib.svgd_linear_backward(dtype, act, n, rows, width, out, Rows(dy, 240, 6), Rows(x, 160, 4), w, ws, z, zn, Rows(dx, *dxs), dw, dws, db, dbs, 0, scratch, sn, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=7), INVALID), (dict(act=9), INVALID), (dict(n=65), TOO_LARGE), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(z=None), INVALID),
    (dict(zn=100), INVALID), (dict(z=B + 4), INVALID), (dict(scratch=None), INVALID), (dict(scratch=S + 8), INVALID), (dict(sn=64), INVALID), (dict(dws=23), INVALID), (dict(db=V + 92), INVALID),
    (dict(db=V + 104), INVALID), (dict(dw=W), INVALID), (dict(dx=Y), INVALID), (dict(dx=X), INVALID), (dict(dx=B), INVALID), (dict(dx=V), INVALID), (dict(dxs=(160, 3)), INVALID), (dict(scratch=U), INVALID),
    (dict(scratch=V), INVALID), (dict(dw=X), INVALID), (dict(db=Y), INVALID), (dict(dw=B), INVALID)])
def test_linear_backward_refuses(lib, bad, status):
    assert linear_backward(lib, **bad) == status


def rotary(**change):
    p = dict(n=2, heads=2, kv_heads=1, dim=8, pairs=4, interleaved=0, batch=2, length=3, frequencies=M, positions=N, positions_stride=3, eps=1e-6, q_weight=W, k_weight=W + 32, q_weight_stride=16,
             k_weight_stride=16)
    return Rotary(**(p | {k: v for k, v in change.items() if k in p}))


QS, KS = (96, 48, 16, 8), (48, 24, 8, 8)


def rotary_forward(lib, dtype=0, q=Q, k=K, qo=O, ko=L, qs=QS, ks=KS, qos=QS, kos=KS, **change):
    return lib.svgd_qk_norm_rotary_forward(dtype, rotary(**change), Heads(q, *qs), Heads(k, *ks), Heads(qo, *qos), Heads(ko, *kos), None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=3), INVALID), (dict(n=0), INVALID), (dict(n=65), TOO_LARGE), (dict(heads=-1), INVALID), (dict(heads=4097), TOO_LARGE), (dict(dim=0), INVALID), (dict(dim=257), TOO_LARGE),
    (dict(pairs=5), INVALID), (dict(pairs=-1), INVALID), (dict(batch=-1), INVALID), (dict(length=-1), INVALID), (dict(length=(1 << 24) + 1), TOO_LARGE), (dict(batch=1 << 20, length=1 << 20), TOO_LARGE),
    (dict(frequencies=None), INVALID), (dict(positions=None), INVALID), (dict(frequencies=M + 4), INVALID), (dict(positions=N + 4), INVALID), (dict(positions_stride=-1), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(q_weight=None), INVALID), (dict(k_weight=None), INVALID), (dict(q_weight=W + 2), INVALID), (dict(q=None), INVALID),
    (dict(ko=None), INVALID), (dict(q=Q + 2), INVALID), (dict(qs=(96, 48, -16, 8)), INVALID), (dict(qos=(96, 48, 16, 7)), INVALID), (dict(qos=(96, 40, 16, 8)), INVALID), (dict(qo=Q + 4), INVALID), (dict(qo=Q), INVALID),
    (dict(qo=K), INVALID), (dict(ko=O), INVALID), (dict(qo=M), INVALID), (dict(qo=N), INVALID), (dict(ko=W), INVALID)])
def test_rotary_forward_refuses(lib, bad, status):
    assert rotary_forward(lib, **bad) == status


def rotary_backward(lib, dtype=0, dqo=O, dko=L, q=Q, k=K, dq=X, dk=Y, dqs=QS, dks=KS, dqw=V, dkw=V + 32, stride=16, scratch=S, sn=1 << 20, **change):
    return lib.svgd_qk_norm_rotary_backward(dtype, rotary(**change), Heads(dqo, *QS), Heads(dko, *KS), Heads(q, *QS), Heads(k, *KS), Heads(dq, *dqs), Heads(dk, *dks), dqw, stride, dkw, stride, 0,
                                            scratch, sn, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=-1), INVALID), (dict(n=65), TOO_LARGE), (dict(dqo=None), INVALID), (dict(q=None), INVALID), (dict(k=K + 1), INVALID), (dict(scratch=None), INVALID), (dict(scratch=S + 4), INVALID),
    (dict(sn=32), INVALID), (dict(stride=7), INVALID), (dict(dqw=W), INVALID), (dict(dkw=V + 16), INVALID), (dict(dq=Q), INVALID), (dict(dq=O + 4), INVALID), (dict(dq=O), INVALID), (dict(dk=X), INVALID), (dict(dk=K), INVALID),
    (dict(scratch=X), INVALID), (dict(scratch=O), INVALID), (dict(dqw=X), INVALID), (dict(dqw=Q), INVALID), (dict(dqw=S), INVALID), (dict(q_weight=None, k_weight=None), INVALID), (dict(dqs=(96, 48, 16, 4)), INVALID)])
def test_rotary_backward_refuses(lib, bad, status):
    assert rotary_backward(lib, **bad) == status


def attention(**change):
    p = dict(n=2, heads=4, kv_heads=2, dim=8, batch=2, length=3, keys=5, causal=1, scale=0.35, cap=0.0, slopes=W, slopes_stride=4, starts=M, lengths=M + 64, documents=M + 128, prefix=M + 512)
    return Attention(**(p | {k: v for k, v in change.items() if k in p}))


AQ, AK = (192, 96, 32, 8), (160, 80, 16, 8)


def attention_forward(lib, dtype=0, q=Q, k=K, v=V, o=O, lse=L, qs=AQ, ks=AK, os=AQ, scratch=S, sn=1 << 24, **change):
    return lib.svgd_attention_forward(dtype, attention(**change), Heads(q, *qs), Heads(k, *ks), Heads(v, *AK), Heads(o, *os), lse, scratch, sn, None)


ATTENTION_BAD = [
    (dict(n=0), INVALID), (dict(n=65), TOO_LARGE), (dict(heads=0), INVALID), (dict(heads=5), INVALID), (dict(kv_heads=0), INVALID), (dict(heads=4098), TOO_LARGE), (dict(heads=514, kv_heads=2), TOO_LARGE),
    (dict(dim=0), INVALID), (dict(dim=129), TOO_LARGE), (dict(batch=-1), INVALID), (dict(batch=(1 << 20) + 1), TOO_LARGE), (dict(length=-1), INVALID), (dict(length=(1 << 24) + 1), TOO_LARGE),
    (dict(length=1 << 24), TOO_LARGE), (dict(keys=-1), INVALID), (dict(keys=(1 << 24) + 1), TOO_LARGE), (dict(batch=1 << 20, keys=1 << 20), TOO_LARGE), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=1e39), INVALID), (dict(scale=float("nan")), INVALID), (dict(cap=-1.0), INVALID), (dict(cap=float("nan")), INVALID), (dict(cap=1e-40), INVALID), (dict(slopes=W + 2), INVALID),
    (dict(starts=M + 2), INVALID), (dict(documents=M + 1), INVALID)]


@pytest.mark.parametrize("bad,status", ATTENTION_BAD + [
    (dict(dtype=3), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(o=None), INVALID), (dict(q=Q + 2), INVALID), (dict(qs=(192, 96, -32, 8)), INVALID),
    (dict(qs=(192, 96, 1 << 23, 8)), TOO_LARGE), (dict(qs=(192, 96, 32, 1 << 22)), TOO_LARGE), (dict(ks=(160, 80, 1 << 23, 8)), TOO_LARGE), (dict(os=(192, 96, 32, 7)), INVALID), (dict(os=(192, 90, 32, 8)), INVALID), (dict(lse=L + 2), INVALID), (dict(o=Q), INVALID),
    (dict(o=K + 4), INVALID), (dict(o=V), INVALID), (dict(lse=Q), INVALID), (dict(lse=O + 8), INVALID), (dict(o=M), INVALID), (dict(lse=M + 128), INVALID), (dict(o=W), INVALID),
    (dict(n=1, batch=1, heads=1, kv_heads=1, keys=4096, scratch=None), INVALID), (dict(n=1, batch=1, heads=1, kv_heads=1, keys=4096, sn=64), INVALID),
    (dict(n=1, batch=1, heads=1, kv_heads=1, keys=4096, scratch=O), INVALID), (dict(n=1, batch=1, heads=1, kv_heads=1, keys=4096, scratch=K), INVALID)])
def test_attention_forward_refuses(lib, bad, status):
    assert attention_forward(lib, **bad) == status


def attention_backward(lib, dtype=0, d_o=X, q=Q, k=K, v=V, o=O, lse=L, dq=Y, dk=U, dv=B, dqs=AQ, dks=AK, ds=R, dss=4, scratch=S, sn=1 << 24, **change):
    return lib.svgd_attention_backward(dtype, attention(**change), Heads(d_o, *AQ), Heads(q, *AQ), Heads(k, *AK), Heads(v, *AK), Heads(o, *AQ), lse, Heads(dq, *dqs), Heads(dk, *dks), Heads(dv, *AK), ds,
                                       dss, 0, scratch, sn, None)


@pytest.mark.parametrize("bad,status", ATTENTION_BAD + [
    (dict(dtype=3), INVALID), (dict(d_o=None), INVALID), (dict(o=None), INVALID), (dict(lse=None), INVALID), (dict(lse=L + 2), INVALID), (dict(scratch=None), INVALID), (dict(scratch=S + 8), INVALID),
    (dict(sn=16), INVALID), (dict(slopes=None), INVALID), (dict(ds=W), INVALID), (dict(dss=3), INVALID), (dict(dq=Q), INVALID), (dict(dq=X), INVALID), (dict(dk=K), INVALID), (dict(dv=V + 4), INVALID),
    (dict(dk=Y), INVALID), (dict(dv=U), INVALID), (dict(dq=L), INVALID), (dict(dk=M), INVALID), (dict(scratch=Y), INVALID), (dict(scratch=L), INVALID), (dict(ds=U), INVALID), (dict(ds=Q), INVALID), (dict(ds=S), INVALID),
    (dict(dqs=(192, 96, 32, 4)), INVALID), (dict(dks=(160, 80, 15, 8)), INVALID)])
def test_attention_backward_refuses(lib, bad, status):
    assert attention_backward(lib, **bad) == status


def test_nothing_to_do(lib):
    assert linear_forward(lib, rows=0, x=None, y=None, z=None, scratch=None) == 0
    assert linear_backward(lib, rows=0, dy=None, x=None, z=None, dx=None, dw=None, db=None, scratch=None) == 0
    assert rotary_forward(lib, batch=0, q=None, k=None, qo=None, ko=None, positions=None, frequencies=None) == 0
    assert rotary_forward(lib, heads=0, kv_heads=0, q=None, k=None, qo=None, ko=None) == 0
    assert rotary_backward(lib, length=0, dqo=None, dko=None, q=None, k=None, dq=None, dk=None, dqw=None, dkw=None, scratch=None) == 0
    assert attention_forward(lib, length=0, q=None, o=None, lse=None) == 0
    assert attention_forward(lib, batch=0, q=None, k=None, v=None, o=None) == 0
    assert attention_backward(lib, batch=0, d_o=None, q=None, k=None, v=None, o=None, lse=None, dq=None, dk=None, dv=None, ds=None, scratch=None, slopes=None) == 0


def test_scratch_sizes(lib):
    assert lib.svgd_linear_saved(2, 3, 5) == 2 * 3 * 8 * 4
    assert lib.svgd_linear_saved(64, 1 << 30, 1 << 20) == 64 * (1 << 50) * 4
    assert lib.svgd_linear_forward_scratch(2, 8, 64, 64) == 0  # few rows
    for bad in ((0, 1, 1, 1), (65, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, 1, 1, (1 << 20) + 1)):
        assert lib.svgd_linear_forward_scratch(*bad) == 0 and lib.svgd_linear_scratch(*bad) == 0
    assert lib.svgd_qk_norm_rotary_scratch(rotary(length=0)) == 0 and lib.svgd_qk_norm_rotary_scratch(rotary(dim=300)) == 0
    assert lib.svgd_attention_forward_scratch(attention()) == 0
    # one token over a cache: parts' sums and their logarithms
    long = attention(n=1, heads=4, kv_heads=1, batch=1, length=1, keys=8192, dim=100)
    parts, rest = divmod(lib.svgd_attention_forward_scratch(long), 4 * 4 * 129)
    assert rest == 0 and parts > 1
    assert lib.svgd_attention_scratch(attention(dim=200)) == 0 and lib.svgd_attention_scratch(attention(slopes=None)) == 2 * 2 * 4 * 3 * 4


def test_python_refuses_what_is_on_no_gpu():
    from paper_2306_06528_amd import attention as att
    x, w, h = torch.zeros(2, 3, 4), torch.zeros(2, 5, 4), torch.zeros(1, 1, 2, 1, 4)
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        att.linear_forward(x, w)
    with pytest.raises(TypeError, match="q must be a CUDA tensor"):
        att.qk_norm_rotary_forward(h, h)
    with pytest.raises(TypeError, match="q must be a CUDA tensor"):
        att.attention_forward(h, h, h)


def test_reference_of_masks():
    """The reference's rule at places that can be seen at a glance."""
    import attention_reference as ref
    see, far = ref.seen(1, 2, 4, causal=True)
    assert see.int().tolist() == [[[1, 1, 1, 0], [1, 1, 1, 1]]] and far.tolist() == [[[2, 1, 0, 1], [3, 2, 1, 0]]]
    ints = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    assert ref.seen(1, 2, 4, causal=True, prefix=ints([4]), lengths=ints([3]))[0].int().tolist() == [[[1, 1, 1, 0], [1, 1, 1, 0]]]
    assert ref.seen(1, 3, 4, starts=ints([-1]), documents=ints([[5, 5, 7, 7]]))[0].int().tolist() == [[[0, 0, 0, 0], [1, 1, 0, 0], [1, 1, 0, 0]]]
