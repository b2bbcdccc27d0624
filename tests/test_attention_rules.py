"""Which instances of the attention kernels a call takes, as far as numbers decide it: compiled for the host and asked."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = r"""
#include <cstdio>
#include "attention_rules.hpp"
using namespace svgd;
struct Sizes { int n, batch, kv, rows, t, s, causal; const int *documents; };
int main()
{
    int size, dim, modified, documents, heads;
    Sizes a;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d", &size, &a.n, &a.batch, &a.t, &a.s, &heads, &a.kv, &dim, &modified, &a.causal, &documents) == 11) {
        a.rows = a.t * (heads / a.kv);
        a.documents = documents ? &documents : nullptr;
        const int kind = dim_kind(dim);
        std::printf("%d %d %d %d %d %d %d\n", kind, few_rows(a), !few_rows(a) && two_forward(size, kind, modified) && many_forward(a), two_keys(size, kind, modified) && many_keys(a), forward_splits(a), query_splits(a),
                    key_splits(a));
    }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not installed")
    d = tmp_path_factory.mktemp("attention_rules")
    (d / "rules.cpp").write_text(PROGRAM)
    csrc = os.path.join(HERE, "..", "paper_2306_06528_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", csrc, "-o", str(d / "rules"), str(d / "rules.cpp")], check=True, timeout=120)

    def ask(calls):
        """calls: (bytes of a value, n, batch, tokens, keys, heads, kv_heads, dim, modified, causal, documents); (kind, few, two in forward, two in keys, forward parts, queries' parts, keys' parts) of each"""
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in calls)
        out = subprocess.run([str(d / "rules")], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


FORWARD = {2: {0, 1, 2, 3, 4}, 4: {0, 1, 2}}  # kinds of heads with two blocks of rows, by bytes of a value
KEYS = {2: {0, 1, 2}, 4: {0, 1}}


def test_the_tests_reach_every_instance_with_two_blocks(rules):
    import test_gpu_attention_two_blocks as two
    for size in (2, 4):
        for sizes, causal in ((two.UNMASKED, False), (two.CAUSAL, True)):
            got = rules([(size, *s, False, causal, False) for s in sizes])
            assert {g[0] for g in got if g[2]} == FORWARD[size] and {g[0] for g in got if g[3]} == KEYS[size]
        assert {g[0] for g in rules([(size, *s, False, True, False) for s in two.LONG]) if g[2]} == FORWARD[size]
        for documents in (False, True):
            got = rules([(size, *s, False, True, documents) for s in two.MASKED])
            assert {g[0] for g in got if g[2]} == FORWARD[size] - {0} and {g[0] for g in got if g[3]} == KEYS[size] - {0}


def test_no_other_instance_has_two(rules):
    calls = [(size, 64, 64, 200, 200, 8, 8, dim, modified, False, False) for size in (2, 4) for dim in (4, 32, 64, 96, 128) for modified in (False, True)]
    for c, (kind, _, forward, keys, *_) in zip(calls, rules(calls)):
        assert forward == (not c[8] and kind in FORWARD[c[0]]) and keys == (not c[8] and kind in KEYS[c[0]])


def test_limits(rules):
    """One workgroup below and at each limit; parts only where workgroups are few, none for one tile."""
    call = lambda batch, s, causal, documents=False: (2, 1, batch, s, s, 1, 1, 64, False, causal, documents)  # noqa: E731
    for s, causal, limit in ((64, False, 1024), (64, True, 4096), (2_048, True, 1536 // 32)):
        assert [g[2] for g in rules([call(limit - 1, s, causal), call(limit, s, causal)])] == [0, 1]
    assert [g[3] for g in rules([call(4_095, 64, False), call(4_096, 64, False), call(4_095, 64, True), call(4_096, 64, True)])] == [0, 1, 0, 1]
    assert rules([call(1, 16, False), call(1, 17, False)])[0][1] == 1 and rules([call(1, 17, False)])[0][1] == 0
    for s in (0, 1, 64, 100, 8_192):
        for batch in (0, 1, 511, 4_096):
            for g in rules([call(batch, s, causal, documents) for causal in (False, True) for documents in (False, True)]):
                tiles = -(-s // 64)
                assert all(1 <= p <= max(1, tiles // 2) for p in g[4:]), (s, batch, g)
    assert all(g[4:] == (1, 1, 1) for g in rules([call(1_024, 8_192, c) for c in (False, True)]))
