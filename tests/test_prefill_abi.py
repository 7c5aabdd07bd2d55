"""Host-side checks of the calls that fill the cache: they come before any launch and need no GPU."""
import ctypes

import pytest
import torch

from paper_2604_09562_amd import binding

P = 1 << 20      # an address that is never read: the checks come first


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_09562_amd import build
        build.build()
    return binding.lib()


def kv(**kw):
    x = binding.ss_paged_kv(10, 16, 8, 128, binding.SS_BF16, P, P, 0, 0)
    for k, v in kw.items():
        setattr(x, k, v)
    return ctypes.byref(x)


def bt(**kw):
    x = binding.ss_batch(4, 8, 0, 0, P, P, P, 0)
    for k, v in kw.items():
        setattr(x, k, v)
    return ctypes.byref(x)


def refused(L, rc, code, text):
    assert rc == code and text in L.ss_last_error(), (rc, L.ss_last_error())


def test_chunk_attention(L):
    def call(c=None, b=None, q=P, stride=4096, dtype=1, hq=32, rows=100, scale=0.1, out=P, ws=P, nbytes=1 << 40):
        return L.ss_chunk_attn(c or kv(), b or bt(), q, stride, dtype, hq, rows, scale, out, None, ws, nbytes, None)
    for kw, code, text in [
        (dict(c=kv(block_size=32)), 1, b"block_size"), (dict(c=kv(head_dim=96)), 1, b"head_dim"), (dict(c=kv(num_kv_heads=5)), 1, b"multiple"),
        (dict(c=kv(dtype=9)), 1, b"dtype"), (dict(c=kv(dtype=2)), 1, b"k_scale"), (dict(c=kv(k_scale=P)), 1, b"k_scale"),
        (dict(c=kv(k=P + 8)), 1, b"aligned"), (dict(c=kv(v=0)), 1, b"NULL"), (dict(c=kv(num_blocks=-1)), 1, b"num_blocks"),
        (dict(c=kv(num_blocks=1 << 27)), 2, b"31 bits"), (dict(c=kv(num_kv_heads=1)), 2, b"16 query heads"), (dict(b=bt(batch=-1)), 1, b"negative"),
        (dict(b=bt(max_blocks_per_seq=0)), 1, b"max_blocks"), (dict(b=bt(max_q_len=-1)), 1, b"max_q_len"), (dict(b=bt(flags=2)), 1, b"flags"),
        (dict(b=bt(tree_mask=P)), 2, b"trees"), (dict(b=bt(kv_len=0)), 1, b"NULL"), (dict(b=bt(max_blocks_per_seq=1 << 28)), 2, b"31 bits"),
        (dict(q=0), 1, b"q is NULL"), (dict(q=P + 2), 1, b"aligned"), (dict(stride=4095), 1, b"apart"), (dict(stride=4100), 1, b"aligned"),
        (dict(dtype=2), 1, b"q_dtype"), (dict(hq=33), 1, b"multiple"), (dict(hq=0), 1, b"multiple"), (dict(rows=-1), 1, b"negative"),
        (dict(rows=1 << 28), 2, b"31 bits"), (dict(scale=0.0), 1, b"sm_scale"), (dict(scale=float("nan")), 1, b"sm_scale"),
        (dict(scale=float("inf")), 1, b"sm_scale"), (dict(out=0), 1, b"NULL"), (dict(out=P + 4), 1, b"out"), (dict(ws=0), 1, b"workspace"),
        (dict(ws=P + 16), 1, b"workspace"), (dict(nbytes=100), 3, b"needed")]:
        refused(L, call(**kw), code, text)
    assert L.ss_chunk_attn(None, bt(), P, 4096, 1, 32, 100, 0.1, P, None, P, 1 << 40, None) == 1
    assert L.ss_chunk_attn(kv(), None, P, 4096, 1, 32, 100, 0.1, P, None, P, 1 << 40, None) == 1
    assert call(rows=0) == 0 and call(b=bt(batch=0)) == 0         # nothing to do, nothing launched


def test_a_scale_whose_powers_of_two_are_no_float(L):
    call = lambda scale: L.ss_chunk_attn(kv(), bt(), P, 4096, 1, 32, 100, scale, P, None, P, 100, None)  # noqa: E731
    refused(L, call(2.5e38), 1, b"sm_scale")
    refused(L, call(-1.0), 1, b"sm_scale")
    refused(L, call(1.9e38), 3, b"needed")               # (the next check's refusal)


def test_chunk_workspace(L):
    size = lambda rows, blocks, dtype=1, **kw: L.ss_chunk_attn_workspace(kv(**kw), bt(max_blocks_per_seq=blocks), dtype, 32, rows)  # noqa: E731
    assert size(100, 8) >= 256 and size(100, 1000) >= size(100, 100) >= size(100, 8)
    assert size(1 << 20, 1000) < 200 << 20                       # bounded, however many rows
    assert size(100, 8, head_dim=80) == 0 and b"head_dim" in L.ss_last_error()
    assert size(100, 8, dtype=7) == 0


def test_kv_write(L):
    def call(c=None, slots=P, k=P, ks=1024, v=P, vs=1024, dtype=1, rows=100):
        return L.ss_kv_write(c or kv(), slots, k, ks, v, vs, dtype, rows, None)
    for kw, code, text in [
        (dict(c=kv(block_size=8)), 1, b"block_size"), (dict(c=kv(head_dim=32)), 1, b"head_dim"), (dict(c=kv(dtype=-1)), 1, b"dtype"),
        (dict(c=kv(dtype=2)), 1, b"k_scale"), (dict(c=kv(dtype=2, k_scale=P)), 1, b"k_scale"), (dict(c=kv(k=0)), 1, b"NULL"),
        (dict(c=kv(v=P + 8)), 1, b"aligned"), (dict(slots=0), 1, b"NULL"), (dict(k=0), 1, b"k_new is NULL"), (dict(v=0), 1, b"v_new is NULL"),
        (dict(k=P + 8), 1, b"k_new"), (dict(ks=1023), 1, b"apart"), (dict(vs=1028), 1, b"v_new"), (dict(vs=-1024), 1, b"apart"),
        (dict(dtype=2), 1, b"new_dtype"), (dict(rows=-1), 1, b"negative"), (dict(rows=1 << 25), 2, b"too large")]:
        refused(L, call(**kw), code, text)
    assert L.ss_kv_write(None, P, P, 1024, P, 1024, 1, 100, None) == 1
    assert call(rows=0) == 0


def test_block_map(L):
    def pool(n=100, ids=P, count=P):
        return ctypes.byref(binding.ss_block_pool(n, ids, count))
    def call(b=None, p=None, held=P, rows=10, slots=P, status=P, ws=P, nbytes=1 << 30):
        return L.ss_block_map(b or bt(), p or pool(), held, rows, slots, None, status, ws, nbytes, None)
    for kw, code, text in [
        (dict(b=bt(batch=-1)), 1, b"negative"), (dict(rows=-1), 1, b"negative"), (dict(b=bt(max_blocks_per_seq=0)), 1, b"max_blocks"),
        (dict(p=pool(n=-1)), 1, b"num_blocks"), (dict(p=pool(n=1 << 27)), 2, b"31 bits"), (dict(p=pool(ids=0)), 1, b"NULL"),
        (dict(p=pool(count=0)), 1, b"NULL"), (dict(held=0), 1, b"NULL"), (dict(slots=0), 1, b"NULL"), (dict(status=0), 1, b"NULL"),
        (dict(b=bt(block_table=0)), 1, b"NULL"), (dict(b=bt(q_indptr=0)), 1, b"NULL"), (dict(ws=0), 1, b"workspace"), (dict(ws=P + 8), 1, b"workspace"),
        (dict(nbytes=8), 3, b"needed")]:
        refused(L, call(**kw), code, text)
    assert L.ss_block_map(None, pool(), P, 10, P, None, P, P, 1 << 30, None) == 1
    assert L.ss_block_map(bt(), None, P, 10, P, None, P, P, 1 << 30, None) == 1
    assert L.ss_block_map_workspace(-1) == 0 and 0 < L.ss_block_map_workspace(0) <= L.ss_block_map_workspace(5000)


def test_rows_of_tensors():
    stride = binding._row_stride
    x = torch.empty(6, 4, 64)
    assert stride(x, 6, 4, 64) == 256 and stride(x[:, :2], 6, 2, 64) == 256 and stride(x[::2], 3, 4, 64) == 512
    for t, args in ((x, (7, 4, 64)), (x, (6, 5, 64)), (x.view(6, 256), (6, 4, 64)), (x.transpose(0, 1), (4, 6, 64)), (x[:, :, ::2], (6, 4, 32)),
                    (torch.empty(6, 64, 4).transpose(1, 2), (6, 4, 64))):
        with pytest.raises(binding.SpecVerifyError):
            stride(t, *args)


def test_tensors_that_are_not_what_an_address_says():
    """Types, lengths and strides are looked at before the library is called; so is the device, on which everything else of these is wrong."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    half = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    base = dict(batch=2, num_q_heads=4, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=6, max_blocks_per_seq=3, total_rows=5, kv_dtype="bf16", q_dtype="bf16",
                new_dtype="bf16", sm_scale=0.1, block_table=i32(2, 3), kv_len=i32(2), q_indptr=i32(3), held=i32(2), free_ids=i32(6), free_count=i32(1),
                k_cache=half(6, 2, 16, 64), v_cache=half(6, 2, 16, 64), k_scale=None, v_scale=None, k_new=half(5, 2, 64), v_new=half(5, 2, 64), q=half(5, 4, 64))
    ws = torch.zeros(1024, dtype=torch.uint8)

    def calls(d, slots=i32(5), positions=i32(5), status=i32(1), out=half(5, 4, 64), lse=torch.zeros(5, 4)):
        binding.ss_block_map(d, slots, positions, status, ws)
        binding.ss_kv_write(d, slots)
        binding.ss_chunk_attn(d, out, lse, ws)

    write = lambda d, slots=i32(5): binding.ss_kv_write(d, slots)  # noqa: E731
    attend = lambda d, out=half(5, 4, 64), lse=torch.zeros(5, 4): binding.ss_chunk_attn(d, out, lse, ws)  # noqa: E731
    long = torch.int64
    for call, text in [
        (lambda: calls(base, slots=i32(5).to(long)), "slot_map .* torch.int64"), (lambda: calls(base, slots=i32(4)), "slot_map .* at least 5"),
        (lambda: calls(base, slots=i32(10)[::2]), "slot_map .*strides"), (lambda: write(base, i32(5).to(long)), "slot_map .* torch.int64"),
        (lambda: write(base, i32(4)), "slot_map .* at least 5"),
        (lambda: write(dict(base, k_new=torch.zeros(5, 2, 64))), "slot_map .* on cpu"),
        (lambda: attend(dict(base, q=torch.zeros(5, 4, 64))), "q must be of type bf16"), (lambda: attend(dict(base, q=half(4, 4, 64))), "expected 5 rows"),
        (lambda: binding.alloc_chunk_outputs(dict(base, block_table=i32(3, 2).T)), "block_table"), (lambda: binding.alloc_block_map_workspace(dict(base, block_table=i32(5))), "block_table"),
        (lambda: binding.alloc_block_map_workspace(base), "block_table .* on cpu"), (lambda: calls(base), "slot_map .* on cpu"), (lambda: attend(base), "q must be .* on cpu")]:
        with pytest.raises(binding.SpecVerifyError, match=text):
            call()
    for check, args, text in [
        (binding._ints, ("x", i32(3).float(), 3), "float32"), (binding._dense, ("x", half(4), 4, 4), "4 bytes"), (binding._dense, ("x", torch.zeros(4, 4).T, 4, 16), "strides"),
        (binding._dense, ("x", torch.zeros(3), 4, 4), "at least 4"), (binding._dense, ("x", torch.zeros(4), 4, 4), "on cpu"), (binding._rows, ("x", torch.zeros(2, 1, 64), "bf16", 2, 1, 64), "type bf16")]:
        with pytest.raises(binding.SpecVerifyError, match=text):
            check(*args)
