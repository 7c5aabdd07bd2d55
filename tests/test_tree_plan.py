"""Host check of how attention of wide draft trees is cut (csrc/chunk_plan.h with the trees' flag): every tile of a request has all of its keys, a request's last tile with half of
the rows or less has cheaper steps, and requests with more new tokens than their masks have bits are left out."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from . import test_chunk_plan as chunks
from .helpers import CSRC

MASK_WORDS = 64


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    text = chunks.SHIM.replace("ss::ChunkWalk<ROWS, KEYS, OPEN> s;", "ss::ChunkWalk<ROWS, KEYS, OPEN, true> s;").replace(
        "args.kv_len = kv_len;", f"args.kv_len = kv_len;\n    args.mask_words = {MASK_WORDS};")
    assert text.count("OPEN, true>") == 1 and text.count("mask_words") == 1
    d = tmp_path_factory.mktemp("tree_plan")
    (d / "shim.cpp").write_text(text)
    subprocess.run(["g++", "-O1", "-std=c++17", "-U_FORTIFY_SOURCE", "-D__HIP_PLATFORM_AMD__", "-shared", "-fPIC", "-isystem", os.path.join(chunks.ROCM, "include"),
                    "-I", os.path.join(chunks.ROOT, "include"), "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = ctypes.CDLL(str(d / "shim.so"))
    lib.plan.restype = ctypes.POINTER(ctypes.c_int32)
    return lib


def check(shim, f32, lengths, hq, hkv, spans):
    rows, keys, G = (64, 64, hq // hkv) if f32 else (256, 32, hq // hkv)
    label = (f32, lengths, hq, hkv, spans)
    tiles, places, cost = {}, {}, {}
    for span, b, t, s0, s1, place, count in chunks.walked(shim, f32, lengths, hq, hkv, spans):
        tiles.setdefault((b, t), []).append((span, s0, s1, place, count))
        left = lengths[b][0] * G - t * rows
        cost[span] = cost.get(span, 0) + (s1 - s0) * (0.75 if left <= rows // 2 else 1.0)
    for b, (q, n) in enumerate(lengths):
        for t in range(-(-q * G // rows)):
            steps = -(-n // keys)
            pieces = tiles.pop((b, t), None)
            assert pieces, (label, b, t, "no piece")
            assert [p[1] for p in pieces] == [0] + [p[2] for p in pieces[:-1]] and pieces[-1][2] == steps, (label, b, t, steps, pieces)
            first = pieces[0][0]
            if len(pieces) == 1:
                assert pieces[0][3] == -1, (label, b, t, pieces)
                continue
            assert pieces[0][4] == len(pieces), (label, b, t, pieces)
            assert [p[3] for p in pieces] == [2 * (first + i) + (i == 0) for i in range(len(pieces))], (label, b, t, pieces)
            for p in pieces:
                assert p[2] > p[1] and p[3] < 2 * spans and p[3] not in places, (label, b, t, pieces)
                places[p[3]] = (b, t)
    assert not tiles, (label, tiles)
    return cost


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 5, 8, 16])
def test_random_batches(shim, f32, G):
    rng = np.random.default_rng(31 * G + f32)
    for _ in range(60):
        hkv = int(rng.choice([1, 2, 4, 8]))
        lengths = []
        for _ in range(int(rng.choice([1, 1, 2, 3, 8, 70]))):
            q = int(round(np.exp(rng.uniform(0, np.log(600)))))
            n = q + (int(np.exp(rng.uniform(0, np.log(20000)))) if rng.random() < 0.7 else 0)
            if rng.random() < 0.1:
                q, n = (0, n) if rng.random() < 0.5 else (q, int(rng.integers(0, q + 1)))   # no new tokens; a cache shorter than the rows
            lengths.append((q, n))
        check(shim, f32, lengths, hkv * G, hkv, int(rng.choice([1, 2, 7, 256 // hkv, 256 // hkv, 512 // hkv])))


@pytest.mark.parametrize("q", [1, 31, 32, 33, 63, 64, 65, 96, 97])
def test_narrow_tiles_are_cut_at_their_cost(shim, q):
    """Rows around half a tile and a whole one (four heads to a KV head)."""
    for batch in (1, 3, 16):
        cost = check(shim, False, [(q, 6000 + 50 * b) for b in range(batch)], 32, 8, 32)
        assert len(cost) == 32 and max(cost.values()) <= 1.1 * sum(cost.values()) / 32 + 20     # (openings cost nine steps, a cut is a step off at most)


def test_more_new_tokens_than_mask_bits(shim):
    most = 32 * MASK_WORDS
    assert {p[1] for p in chunks.walked(shim, False, [(most, most + 50), (most + 1, most + 50), (3, 80)], 8, 2, 16)} == {0, 2}
