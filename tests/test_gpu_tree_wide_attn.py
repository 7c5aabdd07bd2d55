"""ss_tree_attn against the definition in 64 bits: trees of any width, every pair of types, masks of any pattern, empty rows, values that are not finite."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .prefill_ref import DEV, check_chunk

pytestmark = pytest.mark.gpu

MIXED = [(1, 1), (0, 0), (25, 325), (33, 33), (64, 1500), (0, 40), (7, 4000), (130, 131), (1, 17), (40, 56)]
TYPES = [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "fp8")]


# With a bound of the rows short calls take a kernel of their own; without one all of bf16 queries are the other kernel's.
BOTH = pytest.mark.parametrize("most", [None, 0], ids=["bound", "no_bound"])


def run(inp, most=None, lse=True):
    if most is None:
        q = inp["q_indptr"]
        most = int((q[1:] - q[:-1]).max())
    out, l, ws = binding.alloc_tree_outputs(inp, DEV, max_q_len=most)
    out.fill_(7)
    l.fill_(7)
    ws.fill_(0xFF)   # contents are scratch
    binding.ss_tree_attn(inp, out, l if lse else None, ws, max_q_len=most)
    torch.cuda.synchronize()
    used = int(inp["q_indptr"][-1])
    assert (out[used:] == 7).all() and (l[used:] == 7).all(), "rows of no request"
    return out, l


@BOTH
@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 2, 64), (8, 8, 128), (10, 2, 128), (16, 2, 64), (16, 1, 128), (7, 1, 64)])
def test_mixed_batch(q, kv, hq, hkv, d, most):
    inp = ref.tree_batch(MIXED, hq, hkv, d, q=q, kv=kv, seed=hq + d, spare_rows=3, spare_columns=5, spare_words=1, stray_bits=True, row_pad=16)
    ref.check_tree(inp, *run(inp, most))


@BOTH
@pytest.mark.parametrize("q,kv", TYPES[:3])
@pytest.mark.parametrize("pattern", ["tree", "chain", "all", "none", "random"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 1, 64)])
def test_patterns(q, kv, pattern, hq, hkv, d, most):
    lengths = [(31, 31), (32, 64), (65, 200), (96, 96), (5, 5), (1, 1), (257, 700)]
    inp = ref.tree_batch(lengths, hq, hkv, d, pattern=pattern, q=q, kv=kv, seed=3)
    ref.check_tree(inp, *run(inp, most), pattern)


@pytest.mark.parametrize("q,kv", TYPES[:3])
@pytest.mark.parametrize("most", [0, 1, 16, 64, 5000])
def test_any_bound_of_the_rows(q, kv, most):
    """The bound picks a form of the kernel, never the result."""
    inp = ref.tree_batch([(64, 900), (3, 300), (150, 160)], 8, 2, 128, q=q, kv=kv, seed=5)
    ref.check_tree(inp, *run(inp, most))


@BOTH
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129])
@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_every_place_in_a_block(n, kv, most):
    """Trees that begin and end at every place of blocks and steps."""
    inp = ref.tree_batch([(n, n + c) for c in (0, 1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65)], 4, 1, 128, kv=kv, q="f32" if kv == "f32" else "bf16", seed=n)
    ref.check_tree(inp, *run(inp, most))


@BOTH
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_long_and_many(kv, q, most):
    for lengths, hq, hkv in (([(48, 20000)], 8, 2), ([(30, 30 + 37 * i) for i in range(130)], 4, 1), ([(600, 1500)], 4, 4), ([(64, 64 + 5000), (64, 70)], 32, 8)):
        inp = ref.tree_batch(lengths, hq, hkv, 128, kv=kv, q=q, seed=11)
        ref.check_tree(inp, *run(inp, most), str(lengths[:2]))


@BOTH
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_more_nodes_than_positions(kv, q, most):
    """kv_len below the request's rows: nodes in front of position 0 are no keys, and rows that see none are empty."""
    inp = ref.tree_batch([(20, 9), (40, 400), (33, 1), (5, 0)], 8, 2, 128, kv=kv, q=q, pattern="tree", seed=2)
    ref.check_tree(inp, *run(inp, most))


@BOTH
def test_without_log_sum_exp(most):
    for kv, q in (("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")):
        inp = ref.tree_batch(MIXED, 8, 2, 128, kv=kv, q=q, seed=4)
        out, lse = run(inp, most)
        again, untouched = run(inp, most, lse=False)
        assert (untouched == 7).all()
        ref.check_tree(inp, again, lse)


@BOTH
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_chain_is_the_chunks_attention(kv, q, most):
    inp = ref.tree_batch([(70, 300), (33, 2000), (1, 50)], 8, 2, 128, pattern="chain", kv=kv, q=q, seed=6)
    out, lse = run(inp, most)
    check_chunk(inp, out, lse)
    chunk, clse, ws = binding.alloc_chunk_outputs(inp, DEV)
    binding.ss_chunk_attn(inp, chunk, clse, ws)
    ref.check_tree(inp, chunk, clse)


@BOTH
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32"), ("fp8", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("bad", ["key", "value", "both"])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(kv, q, bad, most):
    """Two nodes hold NaN or infinities; rows that do not see them are as if they were not there, the others are not finite."""
    n, m = 90, 400
    inp = ref.tree_batch([(n, m), (30, 60)], 8, 2, 128, kv=kv, q=q, seed=8)
    nodes = (13, 77)
    for node in nodes:
        pos = m - n + node
        block, slot = int(inp["block_table"][0, pos // 16]), pos % 16
        for name in (["k_cache"] if bad == "key" else ["v_cache"] if bad == "value" else ["k_cache", "v_cache"]):
            if kv == "fp8":
                inp[name].view(torch.uint8)[block, :, slot] = 0x7F
            else:
                inp[name][block, :, slot] = float("nan") if name == "k_cache" or node == 13 else float("inf")
    out, lse = run(inp, most)
    sees = inp["sees"][0]
    hit = torch.zeros(inp["total_rows"], dtype=torch.bool)
    for node in nodes:
        hit[:n] |= torch.from_numpy(sees[:, node].copy())
    hit = hit.to(DEV)
    got = (out if out.dtype == torch.float32 else out.view(torch.bfloat16)).float()
    assert not got[hit].isfinite().any()
    clean = dict(inp, k_cache=inp["k_cache"].clone(), v_cache=inp["v_cache"].clone())
    for node in nodes:     # the reference takes other values there: rows that do not see them do not change
        pos = m - n + node
        block, slot = int(inp["block_table"][0, pos // 16]), pos % 16
        for name in ("k_cache", "v_cache"):
            (clean[name].view(torch.uint8) if kv == "fp8" else clean[name])[block, :, slot] = 0
    ref.check_tree(clean, out, lse, rows=(~hit).nonzero()[:, 0])


@BOTH
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_scores_of_any_size(kv, q, most):
    """A scale that takes scores far beyond an exponential's range: the largest score's value, whatever stands in front."""
    for scale in (1e-30, 30.0, 1e12, 1e30):
        inp = ref.tree_batch([(40, 300), (7, 7)], 4, 1, 128, kv=kv, q=q, seed=9)
        inp["sm_scale"] = float(np.float32(scale))
        out, lse = run(inp, most)
        got = (out if out.dtype == torch.float32 else out.view(torch.bfloat16)).double()
        assert got.isfinite().all() and lse.isfinite().all()
        if scale < 1:
            ref.check_tree(inp, out, lse)
            continue
        # weights are one for a row's largest score and nothing elsewhere, where the next one is further away than scores are rounded
        want = torch.full_like(got, float("nan"))
        clear = torch.zeros(got.shape[:2], dtype=torch.bool, device=DEV)
        for b, n in enumerate(inp["kv_len"].tolist()):
            r0, r1 = int(inp["q_indptr"][b]), int(inp["q_indptr"][b + 1])
            k, v = ref.gathered(inp, b, 0, n)
            seen = torch.ones((r1 - r0, n), dtype=torch.bool)
            seen[:, n - (r1 - r0):] = torch.from_numpy(inp["sees"][b])
            x = (inp["q"][r0:r1].double().reshape(-1, 128) @ k.T.contiguous()).view(r1 - r0, 4, n)
            x = torch.where(seen.to(DEV)[:, None], x, -float("inf"))
            top = x.topk(2, -1)
            want[r0:r1] = v[top.indices[..., 0]]
            size = (inp["q"][r0:r1].double().abs().reshape(-1, 128) @ k.abs().T.contiguous()).view(r1 - r0, 4, n).amax(-1)
            gap = top.values[..., 0] - top.values[..., 1]
            clear[r0:r1] = (gap * inp["sm_scale"] > 60) & (gap > 300 * 2.0 ** -24 * size)
        assert clear.float().mean() > (0.02 if scale < 1e3 else 0.9)
        tol = 2.0 ** -8 * want.abs() if q == "bf16" else 2.0 ** -20 * want.abs()
        assert ((got - want).abs() <= tol + 1e-12)[clear].all(), scale


def test_requests_that_cannot_be_are_left_out():
    """Rows outside the call, lengths beyond the table, more nodes than the mask has bits: those rows keep what they hold, the others come out as ever."""
    for kv, q in (("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")):
        inp = ref.tree_batch([(30, 200), (40, 90), (50, 300), (20, 100)], 8, 2, 128, kv=kv, q=q, seed=10)
        good = list(range(30)) + list(range(120, 140))
        broken = dict(inp, kv_len=inp["kv_len"].clone())
        broken["kv_len"][1] = inp["max_blocks_per_seq"] * 16 + 1
        broken["kv_len"][2] = 2 ** 31 - 1
        out, lse = run(broken)
        assert (out[30:120] == 7).all() and (lse[30:120] == 7).all()
        ref.check_tree(inp, out, lse, rows=torch.tensor(good, device=DEV))
        narrow = dict(inp, node_mask=inp["node_mask"][:, :1].contiguous())
        out, lse = run(narrow)
        assert (out[30:120] == 7).all() and (lse[30:120] == 7).all()
        ref.check_tree(inp, out, lse, rows=torch.tensor(good, device=DEV))
        outside = dict(inp, q_indptr=inp["q_indptr"].clone())
        outside["q_indptr"][4] = 10 ** 6
        out, lse, ws = binding.alloc_tree_outputs(outside, DEV)
        out.fill_(7)
        binding.ss_tree_attn(outside, out, lse, ws)
        torch.cuda.synchronize()
        assert (out[120:] == 7).all()
        ref.check_tree(inp, out, lse, rows=torch.arange(120, device=DEV))


def test_block_ids_outside_the_cache_are_not_followed():
    for kv, q in (("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")):
        inp = ref.tree_batch([(30, 200), (40, 90)], 8, 2, 128, kv=kv, q=q, seed=12, garbage=False)
        wild = dict(inp, block_table=inp["block_table"].clone())
        wild["block_table"][1, :6] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, inp["num_blocks"], 5 * 10 ** 8, 0], dtype=torch.int32, device=DEV)
        out, lse = run(wild)
        ref.check_tree(inp, out, lse, rows=torch.arange(30, device=DEV))


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_blocks_behind_four_gigabytes(q):
    """Offsets of keys and values beyond 32 bits."""
    hkv, d, n, m = 8, 128, 40, 700
    inp = ref.tree_batch([(n, m)], 32, hkv, d, q=q, seed=13)
    far = 150000     # blocks of 32 KB
    big = dict(inp, num_blocks=far)
    for name in ("k_cache", "v_cache"):
        big[name] = torch.empty((far, hkv, 16, d), dtype=torch.bfloat16, device=DEV)
        big[name][far - inp["num_blocks"]:] = inp[name]
    big["block_table"] = inp["block_table"] + (far - inp["num_blocks"])
    ref.check_tree(inp, *run(big))


def test_captured_and_on_two_streams():
    """A captured call replayed over new queries, and two calls at once with workspaces of their own, equal the eager ones to the bit."""
    for kv, q in (("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")):
        a = ref.tree_batch([(60, 2000), (25, 300), (0, 0)], 8, 2, 128, kv=kv, q=q, seed=14)
        b = ref.tree_batch([(33, 900)], 8, 2, 128, kv=kv, q=q, seed=15)
        state = [(x, *binding.alloc_tree_outputs(x, DEV, max_q_len=64)) for x in (a, b)]
        eager = [run(x, 64) for x in (a, b)]
        streams = [torch.cuda.Stream() for _ in state]
        for _ in range(3):
            for s, (x, out, lse, ws) in zip(streams, state):
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    binding.ss_tree_attn(x, out, lse, ws, max_q_len=64)
            torch.cuda.synchronize()
            for (x, out, lse, ws), (eo, el) in zip(state, eager):
                assert torch.equal(out, eo) and torch.equal(lse, el)
        x, out, lse, ws = state[0]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.ss_tree_attn(x, out, lse, ws, max_q_len=64)
        for i in range(3):
            if i:
                x["q"].copy_(torch.randn(x["q"].shape, device=DEV).to(x["q"].dtype))
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            eo, el = run(x, 64)
            assert torch.equal(out, eo) and torch.equal(lse, el)


def test_binding_refuses():
    inp = ref.tree_batch([(20, 100)], 8, 2, 128, seed=1)
    out, lse, ws = binding.alloc_tree_outputs(inp, DEV)
    for name, x in (("node_mask", inp["node_mask"].float()), ("node_mask", inp["node_mask"].long()), ("node_mask", inp["node_mask"].cpu()),
                    ("node_mask", inp["node_mask"].repeat(1, 2)[:, ::2]), ("node_mask", inp["node_mask"].view(-1)[:7].contiguous()), ("q", inp["q"].float()),
                    ("q", inp["q"][:, :4]), ("q", inp["q"][:-1])):
        with pytest.raises(binding.SpecVerifyError):
            binding.ss_tree_attn(dict(inp, **{name: x}), out, lse, ws)
    with pytest.raises(binding.SpecVerifyError):
        binding.ss_tree_attn(inp, out[:-1], lse, ws)
    with pytest.raises(binding.SpecVerifyError):
        binding.ss_tree_attn(inp, out, lse.double(), ws)
    with pytest.raises(binding.SpecVerifyError):
        binding.ss_tree_attn(inp, out, lse, ws[:128])
    binding.ss_set_option("validate", 1)
    try:
        with pytest.raises(binding.SpecVerifyError, match="out of range"):
            binding.ss_tree_attn(dict(inp, block_table=inp["block_table"] + 10 ** 6), out, lse, ws)
        binding.ss_tree_attn(inp, out, lse, ws)
    finally:
        binding.ss_set_option("validate", 0)
    ref.check_tree(inp, out, lse)
