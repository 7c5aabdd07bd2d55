"""Refusals of the calls for wide draft trees and shared blocks, and the integer arithmetic of masks: no GPU needed."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .helpers import CSRC


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_09562_amd import build
        build.build()
    return binding.lib()


P = 4096   # an aligned address that nothing follows: refusals come first


def _kv(**kw):
    kv = binding.ss_paged_kv(10, 16, 8, 128, binding.SS_BF16, P, P, 0, 0)
    for k, v in kw.items():
        setattr(kv, k, v)
    return kv


def _bt(**kw):
    bt = binding.ss_batch(4, 8, 0, 0, P, P, P, 0)
    for k, v in kw.items():
        setattr(bt, k, v)
    return bt


def _attn(L, kv=None, bt=None, mask=P, words=2, q=P, stride=32 * 128, dt=1, hq=32, rows=20, scale=0.1, out=P, ws=P, nbytes=1 << 40):
    return L.ss_tree_attn(ctypes.byref(kv or _kv()), ctypes.byref(bt or _bt()), mask, words, q, stride, dt, hq, rows, scale, out, None, ws, nbytes, None)


@pytest.mark.parametrize("code,text,args", [
    (1, b"block_size", dict(kv=_kv(block_size=32))), (1, b"head_dim", dict(kv=_kv(head_dim=96))), (1, b"dtype", dict(kv=_kv(dtype=5))),
    (1, b"multiple", dict(hq=12)), (2, b"16 query heads", dict(hq=8 * 17, stride=8 * 17 * 128)), (1, b"tree_mask", dict(bt=_bt(tree_mask=P))),
    (1, b"negative", dict(bt=_bt(batch=-1))), (1, b"max_blocks", dict(bt=_bt(max_blocks_per_seq=0))), (1, b"max_q_len", dict(bt=_bt(max_q_len=-1))),
    (1, b"flags", dict(bt=_bt(flags=8))), (1, b"mask_words", dict(words=0)), (1, b"mask_words", dict(words=1 << 27)), (1, b"NULL", dict(mask=None)),
    (1, b"NULL", dict(out=None)), (1, b"NULL", dict(bt=_bt(kv_len=0))), (1, b"q is NULL", dict(q=None)), (1, b"elements are", dict(stride=100)),
    (1, b"aligned", dict(stride=32 * 128 + 1)), (1, b"aligned", dict(q=P + 8)), (1, b"aligned", dict(out=P + 4)), (1, b"q_dtype", dict(dt=2)),
    (1, b"sm_scale", dict(scale=0.0)), (1, b"sm_scale", dict(scale=float("nan"))), (1, b"sm_scale", dict(scale=3e38)), (1, b"workspace", dict(ws=None)),
    (1, b"workspace", dict(ws=P + 16)), (3, b"needed", dict(nbytes=0)), (1, b"k_scale", dict(kv=_kv(dtype=binding.SS_FP8_E4M3)))])
def test_tree_attn_refuses(L, code, text, args):
    assert _attn(L, **args) == code and text in L.ss_last_error(), L.ss_last_error()


def test_tree_attn_without_work(L):
    assert _attn(L, bt=_bt(batch=0)) == 0 and _attn(L, rows=0) == 0
    kv, bt = _kv(), _bt(tree_mask=P)
    assert L.ss_tree_attn_workspace(ctypes.byref(kv), ctypes.byref(bt), 1, 32, 20) == 0
    for most in (0, 1, 16, 64, 400):
        bt = _bt(max_q_len=most)
        assert L.ss_tree_attn_workspace(ctypes.byref(kv), ctypes.byref(bt), 1, 32, 20) > 0


def _verify(L, batch=3, vocab=100, stride=104, dt=1, rows=9, depth=0, indptr=P, parent=P, tokens=P, logits=P, u=P, temp=None, t=1.0, n=P, out=P, nodes=P,
            ws=P, nbytes=1 << 40):
    return L.ss_tree_verify(batch, vocab, stride, dt, rows, depth, indptr, parent, tokens, logits, u, temp, t, n, out, nodes, None, ws, nbytes, None)


@pytest.mark.parametrize("code,text,args", [
    (1, b"batch", dict(batch=-1)), (1, b"vocab", dict(vocab=0)), (1, b"max_depth", dict(depth=21)), (1, b"max_depth", dict(depth=-1)), (1, b"row_stride", dict(stride=99)),
    (1, b"logit_dtype", dict(dt=2)), (1, b"temperature", dict(t=-1.0)), (1, b"temperature", dict(t=float("nan"))), (1, b"NULL", dict(indptr=None)),
    (1, b"NULL", dict(parent=None)), (1, b"NULL", dict(tokens=None)), (1, b"NULL", dict(logits=None)), (1, b"NULL", dict(n=None)), (1, b"NULL", dict(out=None)),
    (1, b"NULL", dict(nodes=None)), (1, b"uniforms", dict(u=None)), (1, b"uniforms", dict(u=None, temp=P, t=0.0)), (1, b"aligned", dict(stride=101)),
    (1, b"aligned", dict(logits=P + 2)), (1, b"workspace", dict(ws=None)), (3, b"needed", dict(nbytes=8)), (2, b"too large", dict(batch=1 << 24))])
def test_tree_verify_refuses(L, code, text, args):
    assert _verify(L, **args) == code and text in L.ss_last_error(), L.ss_last_error()


def test_tree_verify_workspace(L):
    assert _verify(L, batch=0) == 0
    assert L.ss_tree_verify_workspace(0, 0, 0) == 0 and L.ss_tree_verify_workspace(-1, 0, 5) == 0
    assert 0 < L.ss_tree_verify_workspace(0, 0, 5) <= L.ss_tree_verify_workspace(4, 40, 5) <= L.ss_tree_verify_workspace(4, 40, 50000)
    assert L.ss_tree_verify_workspace(4, 9, (1 << 30) + 1) == 0 and L.ss_tree_verify_workspace(4, 9, 1 << 30) > 0
    assert _verify(L, vocab=(1 << 30) + 1, stride=(1 << 30) + 8) != 0
    assert L.ss_tree_verify_workspace(4, 1 << 26, 1) < 1 << 16       # more rows than one launch takes: only those on the paths


def _pool(**kw):
    p = binding.ss_block_pool(10, P, P)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _fork(L, bt=None, pool=None, shares=P, held=P, n=2, parent=P, child=P, src=P, dst=P, status=P, ws=P, nbytes=1 << 30):
    return L.ss_block_fork(ctypes.byref(bt or _bt()), ctypes.byref(pool or _pool()), shares, held, n, parent, child, None, src, dst, status, ws, nbytes, None)


def _release(L, bt=None, pool=None, shares=P, held=P, status=P, ws=P, nbytes=1 << 30):
    return L.ss_block_release(ctypes.byref(bt or _bt()), ctypes.byref(pool or _pool()), shares, held, status, ws, nbytes, None)


def _compact(L, bt=None, pool=None, held=P, src=P, dst=P, num=P, status=P, ws=P, nbytes=1 << 30):
    return L.ss_block_compact(ctypes.byref(bt or _bt()), ctypes.byref(pool or _pool()), None, held, None, src, dst, num, status, ws, nbytes, None)


@pytest.mark.parametrize("call", [_fork, _release, _compact])
@pytest.mark.parametrize("code,text,args", [
    (1, b"negative batch", dict(bt=_bt(batch=-1))), (1, b"max_blocks", dict(bt=_bt(max_blocks_per_seq=0))), (1, b"negative num_blocks", dict(pool=_pool(num_blocks=-1))),
    (2, b"31 bits", dict(pool=_pool(num_blocks=1 << 27))), (2, b"2^30", dict(bt=_bt(batch=1 << 20, max_blocks_per_seq=1 << 12))), (1, b"NULL", dict(pool=_pool(free_ids=0))),
    (1, b"NULL", dict(pool=_pool(free_count=0))), (1, b"NULL", dict(held=None)), (1, b"NULL", dict(status=None)), (1, b"NULL", dict(bt=_bt(block_table=0))),
    (1, b"workspace", dict(ws=None)), (1, b"workspace", dict(ws=P + 128)), (3, b"needed", dict(nbytes=4))])
def test_books_refuse(L, call, code, text, args):
    assert call(L, **args) == code and text in L.ss_last_error(), L.ss_last_error()


@pytest.mark.parametrize("code,text,args", [(1, b"num_forks", dict(n=-1)), (2, b"num_forks", dict(n=1 << 21)), (1, b"NULL", dict(parent=None)), (1, b"NULL", dict(child=None)),
                                            (1, b"NULL", dict(src=None)), (1, b"NULL", dict(shares=None)), (1, b"NULL", dict(bt=_bt(kv_len=0)))])
def test_fork_refuses(L, code, text, args):
    assert _fork(L, **args) == code and text in L.ss_last_error(), L.ss_last_error()


def test_release_and_compact_refuse(L):
    assert _release(L, shares=None) == 1 and b"NULL" in L.ss_last_error()
    assert _compact(L, num=None) == 1 and b"NULL" in L.ss_last_error()
    assert _compact(L, dst=None) == 1 and b"NULL" in L.ss_last_error()
    for f, args in ((L.ss_block_fork_workspace, (-1, 0)), (L.ss_block_fork_workspace, (0, -1)), (L.ss_block_release_workspace, (-1, 3, 4)), (L.ss_block_release_workspace, (1, 3, -4)),
                    (L.ss_block_compact_workspace, (-1,))):
        assert f(*args) == 0 and b"negative" in L.ss_last_error()


def test_copy_refuses(L):
    def call(layers, n=2, src=P, dst=P, most=3):
        arr = (binding.ss_paged_kv * len(layers))(*layers)
        return L.ss_block_copy(arr, n, src, dst, most, None, None)
    two = [_kv(), _kv()]
    assert call(two, n=0) == 0 and call(two, most=0) == 0 and call([_kv(num_blocks=0)] * 2) == 0
    assert call(two, n=-1) == 1 and call(two, most=-1) == 1
    assert call(two, src=None) == 1 and call(two, dst=None) == 1
    assert L.ss_block_copy(None, 1, P, P, 1, None, None) == 1
    for other in (_kv(num_blocks=11), _kv(num_kv_heads=4), _kv(head_dim=64), _kv(dtype=binding.SS_F32)):
        assert call([_kv(), other]) == 1 and b"differs" in L.ss_last_error()
    assert call([_kv(), _kv(k=0)]) == 1 and call([_kv(k=P + 8), _kv()]) == 1 and call([_kv(dtype=binding.SS_FP8_E4M3)] * 2) == 1


def test_path_compaction_takes_wide_trees(L):
    """The row bound of ss_kv_compact is gone; ss_kv_append keeps its own."""
    kv, bt = _kv(), _bt(max_q_len=200)
    assert L.ss_kv_compact(ctypes.byref(kv), ctypes.byref(bt), None, None, 4 * 200, None) == 1 and b"NULL" in L.ss_last_error()
    assert L.ss_kv_compact(ctypes.byref(kv), ctypes.byref(bt), None, None, -1, None) == 1 and b"negative" in L.ss_last_error()
    assert L.ss_kv_append(ctypes.byref(kv), ctypes.byref(bt), None, None, 1, 4 * 200, None) == 1 and b"total_rows" in L.ss_last_error()


def test_mask_window(tmp_path):
    """The 32 bits of a row's mask from any node on, for every place of a window and trees of many sizes."""
    text = open(os.path.join(CSRC, "chunk_plan.h")).read()
    body = text[text.index("__device__ __forceinline__ uint32_t tree_window"):]
    body = body[:body.index("\n}\n") + 3].replace("__device__ __forceinline__", 'extern "C"')
    src, lib = tmp_path / "w.cpp", tmp_path / "w.so"
    src.write_text("#include <stdint.h>\n" + body)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    fn = ctypes.CDLL(str(lib)).tree_window
    fn.restype, fn.argtypes = ctypes.c_uint32, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    rng = np.random.default_rng(0)
    for words in (1, 2, 3):
        for q_len in (1, 2, 31, 32, 33, 63, 64, 65, 96):
            if q_len > words * 32:
                continue
            row = rng.integers(0, 2, words * 32).astype(bool)
            packed = np.ascontiguousarray(ref.pack(row[None], words)[0])
            for n0 in range(-70, 130):
                want = [n < 0 or (n < q_len and row[n]) for n in range(n0, n0 + 32)]
                got = fn(packed.ctypes.data, words, q_len, n0)
                assert [(got >> i) & 1 == 1 for i in range(32)] == want, (words, q_len, n0)
