"""Which tiles the gated feed-forward block takes, as far as numbers decide it: compiled for the host and asked."""
import collections
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
TOO_LARGE = -3

PROGRAM = r"""
#include <cstdio>
#include "ffn_rules.hpp"
using namespace svgd;
int main()
{
    long long n, rows, width, hidden;
    while (std::scanf("%lld %lld %lld %lld", &n, &rows, &width, &hidden) == 4) {
        const ForwardPlan f((int)n, rows, width, hidden);
        const BackwardPlan b((int)n, rows, width, hidden, true);
        const auto count = [&](TileKind k, long long i, long long j, int per_i) { return (long long)(n * tiles(i, kKinds[k].i / per_i) * tiles(j, kKinds[k].j)); };
        const TileKind g = b.gradients;
        std::printf("%d %d %d %lld %d %d %lld %d %d %d %lld %d %d %d %lld %d %d\n", f.fits(), f.thin, f.gate_up.kind, count(f.gate_up.kind, hidden, rows, 2), f.down.kind,
                    f.down.parts, count(f.down.kind, width, rows, 1) * f.down.parts, b.fits(), b.thin, b.hidden.kind, count(b.hidden.kind, hidden, rows, 1), g,
                    b.input_parts, b.param_parts,
                    (b.thin_input ? 0 : count(g, width, rows, 1) * b.input_parts) + 3 * count(g, width, hidden, 1) * b.param_parts, b.thin_input,
                    BackwardPlan((int)n, rows, width, hidden, false).thin_input);
    }
}
"""
THREADS = (256, 128, 64)
Plan = collections.namedtuple("Plan", "fits thin gate_up gate_up_tiles down down_parts down_tiles back_fits back_thin dh dh_tiles gradients input_parts param_parts "
                              "gradients_tiles dx_thin dx_alone_thin")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not installed")
    d = tmp_path_factory.mktemp("ffn_rules")
    (d / "rules.cpp").write_text(PROGRAM)
    csrc = os.path.join(HERE, "..", "paper_2306_06528_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", csrc, "-o", str(d / "rules"), str(d / "rules.cpp")], check=True, timeout=120)

    def ask(shapes):
        text = "".join("%d %d %d %d\n" % s for s in shapes)
        out = subprocess.run([str(d / "rules")], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [Plan(*map(int, line.split())) for line in out.splitlines()]
    return ask


def launches(p):
    """(kind, tiles) of every launch that is one of tiles."""
    forward = [] if p.thin else [(p.gate_up, p.gate_up_tiles), (p.down, p.down_tiles)]
    return forward + ([] if p.back_thin else [(p.dh, p.dh_tiles)]) + [(p.gradients, p.gradients_tiles)]


def test_narrow_layers_of_very_many_rows_take_tiles_that_a_launch_takes(rules):
    """Layers whose fastest tiles would be small ones, more than a launch of 2^32 threads has, and that fit the card."""
    shapes = [(1, 600_000_000, 8, 32), (1, 1 << 30, 1, 8), (64, 16_000_000, 4, 16), (1, 700_000_000, 16, 32), (4, 250_000_000, 8, 8), (16, 60_000_000, 30, 40)]
    for shape, p in zip(shapes, rules(shapes)):
        assert p.fits and p.back_fits, shape
        # (up to three grids of a launch, each filled up to a multiple of eight)
        assert all((count + 21) * THREADS[kind] < 1 << 32 for kind, count in launches(p)), shape


def test_more_tiles_than_a_launch_takes_are_refused_before_the_first_launch(rules):
    shapes = [(64, 1 << 30, 1, 1), (64, 1 << 20, 1 << 20, 1 << 20), (64, 1, 1 << 20, 1 << 20)]
    assert [(p.fits, p.back_fits) for p in rules(shapes)] == [(False, False), (False, False), (True, False)]
    from test_layers_cpu import Library
    lib = Library()
    n, rows, width, hidden = shapes[0]
    x, gate, up, down, y, buffer, dx, dgate, dup, ddown, scratch = (k << 56 for k in range(1, 12))  # made-up addresses, 2^56 bytes apart
    act = lambda p: lib._Rows(p, rows * width, width)
    size = width * hidden
    assert lib._lib.svgd_gated_ffn_forward(0, 0, n, rows, width, hidden, act(x), gate, size, up, size, down, size, act(y), 1, buffer, 1 << 50, scratch, 1 << 50, None) == TOO_LARGE
    assert lib._lib.svgd_gated_ffn_backward(0, 0, n, rows, width, hidden, act(y), act(x), gate, size, up, size, down, size, buffer, 1 << 50, act(dx), dgate, size,
                                            dup, size, ddown, size, 0, scratch, 1 << 50, None) == TOO_LARGE


def test_every_plan_of_up_to_256_gib_can_be_launched(rules):
    rng = random.Random(5)
    between = lambda low, high: int(round(low * (high / low) ** rng.random()))
    shapes = []
    while len(shapes) < 4000:
        n, rows, width, hidden = between(1, 64), between(1, 1 << 30), between(1, 1 << 20), between(1, 1 << 20)
        if n * (rows * (4 * width + 4 * (-(-hidden // 32) * 32)) + 12 * width * hidden) < 256 << 30:  # x and y of 16 bits, h, the parameters
            shapes.append((n, rows, width, hidden))
    for shape, p in zip(shapes, rules(shapes)):
        assert p.fits and p.back_fits, shape
        assert all((count + 21) * THREADS[kind] < 1 << 32 for kind, count in launches(p)), shape
        assert p.input_parts == 1 or p.input_parts % 2 == 0
        assert p.down_parts <= max(1, shape[3] // 128) and p.param_parts <= max(1, shape[1] // 128)


def test_the_shapes_that_are_tested_reach_every_tile(rules):
    """Every kind of tile in every product, in one part and in several, with at least three whole steps and a part of one in each."""
    from ffn_shapes import TILES
    seen = set()
    for (n, rows, width, hidden), p in zip(TILES, rules(TILES)):
        steps = lambda columns, parts: columns // parts >= 96 and columns % 32
        if not p.thin:
            if steps(width, 1):
                seen |= {("gate_up", p.gate_up)}
            if steps(hidden, p.down_parts):
                seen |= {("down", p.down, p.down_parts > 1)}
            if rows <= 64:
                seen |= {("33 to 64 rows", p.gate_up)}
        if steps(width, 1):
            seen |= {("dh", p.dh)}
        if steps(hidden, max(1, p.input_parts // 2)) and steps(rows, p.param_parts):
            seen |= {("gradients", p.gradients, p.input_parts > 1, p.param_parts > 1)}
    want = {(what, kind) for what in ("gate_up", "dh") for kind in range(3)} | {("down", kind, parts) for kind in range(3) for parts in (False, True)}
    want |= {("gradients", kind, a, b) for kind in range(3) for a in (False, True) for b in (False, True)}
    want |= {("33 to 64 rows", kind) for kind in (1, 2)}
    assert want <= seen, want - seen


def test_the_shapes_that_are_tested_give_waves_of_few_rows_several_steps(rules):
    """Eight waves take turns over steps of 32 columns: two steps at once, a third one by itself, and a part of a step behind whole ones."""
    from ffn_shapes import THIN
    seen = set()
    for (n, rows, width, hidden), p in zip(THIN, rules(THIN)):
        assert p.thin
        if all(columns // 32 // 8 >= 2 and -(-(columns // 32) // 8) % 2 == 1 and columns % 32 for columns in (width, hidden)):
            seen |= {(rows > 16) + (rows > 32)}
    assert seen == {0, 1, 2}


def test_the_shapes_that_are_tested_take_every_way_to_dx_of_few_rows(rules):
    from ffn_shapes import DX_OF_FEW_ROWS, THIN
    plans = rules(DX_OF_FEW_ROWS + THIN)
    assert all(p.back_thin for (_, rows, *_), p in zip(DX_OF_FEW_ROWS + THIN, plans) if rows <= 32)
    assert {(rows > 16, p.dx_thin, p.dx_alone_thin) for (_, rows, *_), p in zip(DX_OF_FEW_ROWS, plans)} == {
        (more, a, b) for more in (False, True) for a, b in ((0, 0), (0, 1), (1, 0), (1, 1))}
    assert {p.gradients for (_, rows, *_), p in zip(DX_OF_FEW_ROWS + THIN, plans) if rows <= 32} == {1, 2}
    # (the longest way: a wave goes through all of the hidden width for dx)
    assert not any(p.dx_alone_thin for p in rules([(1, 1, 256, 16_000), (1, 32, 16, 1 << 20)]))
    assert all(p.dx_thin and p.dx_alone_thin for p in rules([(n, 0, width, hidden) for n in (1, 64) for width in (1, 700) for hidden in (1, 5_000)]))
