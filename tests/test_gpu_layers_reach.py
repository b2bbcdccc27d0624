"""The particles' layers where sizes lead the kernels to ways that the other tests' sizes do not."""
import pytest
import torch

import layer_reference as ref
from test_gpu_layers import IDS, TYPES, acts, gen, layers, params, run_ffn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_ffn_more_small_tiles_than_a_launch_takes(layers):  # noqa: F811
    """600 million rows of a narrow layer, 77 GB of h: the fastest tiles would be 18.75 million."""
    rows, width, hidden = 600_000_000, 8, 32
    x = torch.rand(1, rows, width, generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16) - 0.5
    p, _, _, _ = params(gen(41), 1, 3, (hidden, width), (hidden, width), (width, hidden), spread=0.5)
    y, _ = layers.gated_ffn_forward(x, *p)
    for first in (0, rows // 2 - 7, (1 << 26) * 8 - 20, rows - 40):  # (the third: where x's values pass 2^32)
        part = slice(first, first + 40)
        ref.check(y[:, part], ref.gated_ffn(x[:, part], *p, "silu")["y"], f"y from row {first} on")
