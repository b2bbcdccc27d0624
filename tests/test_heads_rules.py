"""Whether tensors with heads meet in memory, as far as numbers decide it: compiled for the host, asked, and compared with sets of addresses."""
import itertools
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = r"""
#include <cstdio>
#include "heads_rules.hpp"
using namespace svgd;
int main()
{
    long long size, v[2][10];
    while (std::scanf("%lld", &size) == 1) {
        svgd_heads h[2];
        HeadSizes s[2];
        for (int i = 0; i < 2; ++i) {
            for (long long &x : v[i])
                if (std::scanf("%lld", &x) != 1) return 1;
            h[i] = {(void *)v[i][0], v[i][1], v[i][2], v[i][3], v[i][4]};
            s[i] = {v[i][5], v[i][6], v[i][7], v[i][8], v[i][9]};
        }
        std::printf("%d\n", heads_apart(h[0], s[0], h[1], s[1], size));
    }
}
"""


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not installed")
    d = tmp_path_factory.mktemp("heads_rules")
    (d / "rules.cpp").write_text(PROGRAM)
    csrc = os.path.join(HERE, "..", "paper_2306_06528_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", csrc, "-o", str(d / "rules"), str(d / "rules.cpp")], check=True, timeout=120)

    def ask(pairs, size=2):
        text = "".join(f"{size} {' '.join(map(str, a))} {' '.join(map(str, b))}\n" for a, b in pairs)
        out = subprocess.run([str(d / "rules")], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [bool(int(line)) for line in out.split()]
    return ask


AT = 1 << 20


def parts(n, batch, tokens, counts, dim, order="nbth", pad=0):
    """Views of so many heads each, one behind the other, of one buffer whose dimensions follow one another as `order` says."""
    total = sum(counts)
    sizes = {"n": n, "b": batch, "t": tokens, "h": total}
    strides, step = {}, dim + pad
    for name in reversed(order):
        strides[name] = step
        step *= sizes[name]
    out, first = [], 0
    for c in counts:
        out.append((AT + 2 * first * strides["h"], strides["n"], strides["b"], strides["t"], strides["h"], n, batch, tokens, c, dim))
        first += c
    return out


def addresses(h, size=2):
    data, *rest = h
    strides, sizes = rest[:4], rest[4:8]
    return {data // size + sum(s * i for s, i in zip(strides, at)) + c for at in itertools.product(*map(range, sizes)) for c in range(h[-1])}


@pytest.mark.parametrize("order", ["".join(p) for p in itertools.permutations("nbth")])
@pytest.mark.parametrize("sizes", [(2, 3, 5), (1, 2, 4), (3, 1, 2), (2, 2, 1), (1, 1, 7)])
def test_parts_of_one_buffer(apart, order, sizes):
    """dq, dk and dv of one dqkv, whatever lies inside of what."""
    q, k, v = parts(*sizes, (4, 2, 2), 8, order, pad=3)
    assert apart([(q, k), (k, q), (q, v), (v, k)]) == [True] * 4
    nearer = (k[0] - 2, *k[1:])  # one value into the queries' last head, or into what is between heads
    assert apart([(q, nearer), (q, q), (nearer, nearer)])[1:] == [False, False]
    assert apart([(q, nearer)])[0] <= (not addresses(q) & addresses(nearer))


def test_what_is_said_apart_is(apart):
    """Random pairs in one small buffer: never said apart where they have an address in common, and said so where they are parts of one buffer."""
    rng = random.Random(5)
    pairs = []
    for _ in range(6_000):
        h = parts(rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3), [rng.randint(1, 3) for _ in range(3)], rng.randint(1, 5), "".join(rng.sample("nbth", 4)), rng.randint(0, 3))
        a, b = (list(x) for x in rng.sample(h, 2))
        for x in (a, b):
            if rng.random() < 0.5:
                x[rng.randint(1, 4)] += rng.choice([-3, -1, 1, 2, 7, 30])
            if rng.random() < 0.3:
                x[0] += 2 * rng.randint(-6, 6)
            if rng.random() < 0.3:
                x[rng.randint(5, 8)] = rng.randint(1, 4)
        if min(a[1:5] + b[1:5]) >= 0:
            pairs.append((tuple(a), tuple(b)))
    said = apart(pairs)
    for (a, b), yes in zip(pairs, said):
        if yes:
            assert not addresses(a) & addresses(b), (a, b)
    assert sum(said) > 1_000 and sum(not s for s in said) > 1_000


def test_nothing_meets_nothing(apart):
    q, k = parts(2, 2, 3, (2, 2), 4)
    empty = (*k[:7], 0, *k[8:])
    assert apart([(q, (0, *k[1:])), (q, empty), (q, (q[0], *empty[1:]))]) == [True] * 3
