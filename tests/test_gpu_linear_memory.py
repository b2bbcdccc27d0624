"""Scratch memory of the linear map's backward pass: dz, as large as twice dy, is in it only where there is an activation."""
import pytest
import torch

from test_attention_cpu import Rows, lib  # noqa: F401
from test_gpu_attention import gen, normal, params

pytestmark = pytest.mark.gpu
NONE, INVALID = 4, -1


@pytest.fixture(scope="module")
def att():
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2306_06528_amd import attention as mod
    return mod


@pytest.mark.parametrize("n,rows,width,out", [(2, 600, 64, 130), (1, 5, 7, 3), (3, 1_500, 33, 40), (8, 1_576, 384, 500)])
def test_without_an_activation_dz_takes_none(att, lib, n, rows, width, out):  # noqa: F811
    g = gen("memory", rows)
    x, dy = normal(g, n, rows, width, dtype=torch.bfloat16), normal(g, n, rows, out, dtype=torch.bfloat16)
    (w, b), (dw, db), G, _ = params(g, n, 0, (out, width), (out,))
    want = att.linear_backward(dy, x, w, None, dw, db)
    grads = G.clone()
    size = lib.svgd_linear_scratch(n, rows, width, out) - lib.svgd_linear_saved(n, rows, out)
    memory = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)

    def call(size):
        return lib.svgd_linear_backward(1, NONE, n, rows, width, out, Rows(dy.data_ptr(), rows * out, out), Rows(x.data_ptr(), rows * width, width), w.data_ptr(), w.stride(0), None, 0,
                                        Rows(dx.data_ptr(), rows * width, width), dw.data_ptr(), dw.stride(0), db.data_ptr(), db.stride(0), 0, memory.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    assert call(size - 1) == INVALID
    G.fill_(-7.0)
    assert call(size) == 0
    assert torch.equal(dx, want) and torch.equal(G, grads) and (memory[size:] == 77).all()


def test_what_a_call_allocates(att):
    n, rows, width, out = 4, 8_192, 64, 512
    x, dy, w = (torch.zeros(*s, device="cuda", dtype=t) for s, t in (((n, rows, width), torch.float16), ((n, rows, out), torch.float16), ((n, out, width), torch.float32)))
    dw = torch.empty_like(w)

    def peak(activation, saved):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        att.linear_backward(dy, x, w, saved, dw, None, activation)
        return torch.cuda.max_memory_allocated() - before
    saved = att.linear_forward(x, w, activation="silu", save=True)[1]
    assert peak("silu", saved) - peak("none", None) >= n * rows * out * 4 - 4096
