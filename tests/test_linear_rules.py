"""Which tiles a linear map takes, as far as numbers decide it: compiled for the host and asked."""
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = r"""
#include <cstdio>
#include "linear_rules.hpp"
using namespace svgd;
int main()
{
    long long n, rows, width, out;
    while (std::scanf("%lld %lld %lld %lld", &n, &rows, &width, &out) == 4) {
        const LinearForwardPlan f((int)n, rows, width, out);
        const LinearBackwardPlan b((int)n, rows, width, out);
        std::printf("%d %d %d %d %d %d %d %d %d %lld %zu\n", f.fits(), f.thin, f.tile.kind, f.tile.parts, b.fits(), b.kind, b.input_parts, b.param_parts, b.sums, (long long)b.sum_rows, b.scratch());
    }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not installed")
    d = tmp_path_factory.mktemp("linear_rules")
    (d / "rules.cpp").write_text(PROGRAM)
    csrc = os.path.join(HERE, "..", "paper_2306_06528_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", csrc, "-o", str(d / "rules"), str(d / "rules.cpp")], check=True, timeout=120)

    def ask(shapes):
        text = "".join("%d %d %d %d\n" % s for s in shapes)
        out = subprocess.run([str(d / "rules")], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_the_tests_shapes_take_every_kind(rules):
    """What test_gpu_attention.py runs: few rows; every kind of tile forward and backward, with the columns whole and in parts."""
    from test_gpu_attention import LINEAR_SIZES
    plans = rules([*LINEAR_SIZES, (8, 1_576, 384, 1_153), (4, 2_050, 1_030, 1_029), (20, 333, 500, 500), (2, 3_001, 97, 600)])
    forward = {(p[2], p[3] > 1) for p in plans if not p[1]}
    backward = {p[5] for p in plans}
    assert any(p[1] for p in plans)
    assert {k for k, _ in forward} == {0, 1, 2} and any(parts for _, parts in forward), forward
    assert backward == {0, 1, 2} and any(p[6] > 1 for p in plans) and any(p[7] > 1 for p in plans) and any(p[8] > 1 for p in plans), backward


def test_parts_cover_the_rows(rules):
    rng = random.Random(1)
    shapes = [(rng.randint(1, 64), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 11))) for _ in range(3000)]
    for (n, rows, width, out), p in zip(shapes, rules(shapes)):
        fits, thin, kind, parts, back_fits, back_kind, ip, pp, sums, per, scratch = p
        assert fits and back_fits and parts >= 1 and ip >= 1 and pp >= 1
        assert (sums - 1) * per < rows <= sums * per and 1 <= sums <= 128
        assert parts == 1 or width // parts >= 128
        floats = n * rows * ((out + 3) // 4 * 4) + (ip > 1) * ip * n * rows * ((width + 3) // 4 * 4) + (pp > 1) * pp * n * width * out + (sums > 1) * sums * n * out
        assert scratch >= 4 * floats


def test_no_rows(rules):
    for p in rules([(1, 0, 5, 7), (64, 0, 1, 1 << 20)]):
        assert p[8] == 0 and p[7] == 1
