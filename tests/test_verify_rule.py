"""Which form the verification of trees takes, and the workspace that it asks for: the rule, compiled for the host, and the sizes by the C ABI; no GPU needed."""
import ctypes
import os
import subprocess

import pytest

from paper_2604_09562_amd import binding

from .helpers import CSRC

DEEPEST = 20


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "r.cpp").write_text('#include "tree_verify_rule.h"\n'
                             'extern "C" int all_rows(int b, long long rows, int vocab, int depth) { return ss::verify_all_rows(b, rows, vocab, depth); }\n'
                             'extern "C" long long most(int b, int vocab, int depth) { return ss::verify_most_rows(b, vocab, depth); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    r = ctypes.CDLL(str(d / "r.so"))
    r.all_rows.argtypes = [ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    r.most.argtypes, r.most.restype = [ctypes.c_int] * 3, ctypes.c_longlong
    return r


@pytest.fixture(scope="module")
def size():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_09562_amd import build
        build.build()
    return binding.lib().ss_tree_verify_workspace


VOCABS = [1, 100, 2049, 5000, 32000, 128256, 152064, 600_001, 1 << 30]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("batch", [1, 3, 64, 1000, 60000])
def test_the_most_rows_that_are_taken_at_once(rule, batch, vocab):
    for depth in (1, 4, 8, DEEPEST):
        most = rule.most(batch, vocab, depth)
        assert most == 0 or rule.all_rows(batch, most, vocab, depth)
        assert not rule.all_rows(batch, most + 1, vocab, depth)
        assert most <= rule.most(batch, vocab, DEEPEST)
    fours = -(-vocab // 8192)
    assert not rule.all_rows(batch, -(-(1 << 23) // fours), vocab, DEEPEST)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("batch", [1, 3, 64, 1000])
def test_a_workspace_serves_every_smaller_step(size, batch, vocab):
    """One for the largest step is one for those with fewer rows or requests, on both sides of the rule's border."""
    rows = sorted({0, 1, 2, 40, 130, 800, 3200, 3300, 4096} | {round(1.3 ** i) for i in range(60)})
    rows = [r for r in rows if r * -(-vocab // 8192) < 1 << 23]
    sizes = [size(batch, r, vocab) for r in rows]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))
    for less in {1, batch // 2, batch - 1} - {0}:
        assert all(size(less, r, vocab) <= s for r, s in zip(rows, sizes))


def test_workspaces_stay_small(size):
    for vocab in (5000, 32000, 128256, 600_001):
        assert size(1, 1 << 13, vocab) < 1 << 20 and size(64, 1 << 13, vocab) < 1 << 20


def test_the_cases_of_rounds_are_taken_in_rounds(rule):
    from .test_gpu_tree_rounds import SHAPES
    for nodes, vocab, depth in SHAPES.values():
        assert not rule.all_rows(len(nodes), sum(nodes), vocab, depth or DEEPEST)


def test_few_rows_are_taken_at_once_and_many_are_not(rule):
    assert rule.all_rows(1, 25, 32000, 6) and rule.all_rows(64, 64 * 12, 32000, 8) and rule.all_rows(64, 64, 128256, 20)
    assert not rule.all_rows(64, 64 * 40, 128256, 8) and not rule.all_rows(20000, 60000, 1000, 8) and not rule.all_rows(1000, 48000, 100, 8)
