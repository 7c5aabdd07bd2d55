"""ss_chunk_attn against attention in 64 bits, within bounds that follow from the roundings."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding
from tests import prefill_ref as ref

pytestmark = pytest.mark.gpu


def run(inp, lse=True, label=""):
    out, z, ws = binding.alloc_chunk_outputs(inp)
    out.view(torch.uint8).fill_(0x5A)
    z.fill_(123.0)
    ws.fill_(0xFF)                               # what a workspace holds is of no account
    binding.ss_chunk_attn(inp, out, z if lse else None, ws)
    torch.cuda.synchronize()
    used = int(inp["q_indptr"][-1])
    assert (out.view(torch.uint8)[used:] == 0x5A).all() and (z[used:] == 123.0).all(), "rows of no request are left as they were"
    if not lse:
        assert (z == 123.0).all()
        z = ref.chunk_reference(inp)[1].float()
    ref.check_chunk(inp, out, z, label)
    return out, z


# one token to many, lengths on both sides of blocks (16), steps (64) and tiles, requests without rows or without a cache
EDGES = [(1, 1), (1, 16), (1, 17), (2, 2), (15, 15), (16, 16), (17, 17), (31, 63), (32, 64), (33, 65), (63, 64), (64, 64), (65, 65), (1, 640),
         (0, 0), (0, 50), (127, 130), (128, 128), (129, 300)]


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "fp8")])
@pytest.mark.parametrize("d", [64, 128])
def test_edge_lengths(q, kv, d):
    run(ref.chunk_batch(EDGES, 8, 2, d, kv, q, seed=d, spare_rows=5, spare_columns=2))


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (4, 2), (6, 2), (5, 1), (14, 2), (16, 2), (32, 8), (16, 1), (26, 2)])
def test_head_groupings(q, kv, hq, hkv):
    run(ref.chunk_batch([(40, 100), (1, 70), (97, 97), (3, 300)], hq, hkv, 128, kv, q, seed=hq))


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("lengths", [[(700, 700)], [(300, 2100)], [(64, 5000)], [(1, 9000)], [(130, 1500), (1, 4000), (500, 500), (7, 20)]],
                         ids=["prompt", "last_piece", "few_rows_long_cache", "one_row", "mixed"])
def test_long(q, kv, lengths):
    run(ref.chunk_batch(lengths, 8, 2, 128, kv, q, seed=len(lengths)))


def test_the_same_table_wider_and_without_lse():
    for extra in (0, 1, 50, 3000):
        run(ref.chunk_batch([(90, 333), (5, 900)], 8, 2, 128, spare_columns=extra, seed=4), lse=False)


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_rows_that_see_nothing(q, kv):
    """A cache shorter than the request's rows: the first rows are in front of it."""
    lengths = [(40, 40), (30, 10), (20, 0), (200, 130), (1, 0)]
    inp = ref.chunk_batch(lengths, 8, 2, 64, kv, q, seed=9)
    out, z = run(inp)
    assert torch.isinf(z[40:60]).all() and (out[40:60] == 0).all() and torch.isfinite(z[60:70]).all()


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("f32", "f32")])
def test_queries_in_wider_rows(q, kv):
    inp = ref.chunk_batch([(50, 120), (1, 30)], 8, 2, 128, kv, q, row_pad=264, seed=2)
    a, za = run(inp)
    dense = dict(inp, q=inp["q"].contiguous())
    b, zb = run(dense)
    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(za, zb)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_sharp_and_flat_scores(kv):
    for sharp in (0.0, 0.01, 30.0):
        run(ref.chunk_batch([(70, 400), (200, 200)], 4, 1, 128, kv, sharp=sharp, seed=6), label=f"sharp {sharp}")


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("f32", "f32")])
def test_scores_that_grow_along_the_cache(q, kv):
    """Each step's largest score is far above the last one's, and the other way round."""
    for sign in (1.0, -1.0):
        inp = ref.chunk_batch([(90, 700)], 4, 1, 128, kv, q, seed=8)
        n = 700
        ids = inp["block_table"][0].long()
        ramp = torch.arange(ids.numel() * 16, device="cuda").view(-1, 16).float() / n * 40.0 * sign
        k = torch.zeros_like(inp["k_cache"])
        k[ids, 0, :, 0] = ramp.to(k.dtype)
        inp["k_cache"] = k
        inp["q"] = inp["q"].clone()
        inp["q"][:, :, 0] = 11.25
        run(inp, label=f"ramp {sign}")


def test_negative_and_zero_scales():
    inp = ref.chunk_batch([(90, 300), (3, 40)], 8, 2, 128, "fp8", seed=12)
    inp["k_scale"][::3] *= -1.0
    inp["v_scale"][1::4] = 0.0
    run(inp)


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("fp8", 128), ("bf16", 64)])
def test_what_later_rows_see_may_be_infinite(kv, d):
    """A key or value that is not finite reaches the rows that see it and no other."""
    inp = ref.chunk_batch([(150, 200)], 4, 1, d, kv, seed=3)
    clean = dict(inp, k_cache=inp["k_cache"].clone(), v_cache=inp["v_cache"].clone())
    pos = 120                                            # seen from row 70 on
    blk, place = int(inp["block_table"][0, pos // 16]), pos % 16
    for name in ("k_cache", "v_cache"):
        raw = inp[name].view(torch.uint8) if kv == "fp8" else inp[name]
        raw[blk, 0, place, 5] = 0x7F if kv == "fp8" else float("inf") if name == "v_cache" else float("nan")
    out, z, ws = binding.alloc_chunk_outputs(inp)
    binding.ss_chunk_attn(inp, out, z, ws)
    want, zw, _ = binding.alloc_chunk_outputs(clean)
    binding.ss_chunk_attn(clean, want, zw, ws)
    torch.cuda.synchronize()
    assert torch.equal(out[:70], want[:70]) and torch.equal(z[:70], zw[:70])
    assert not torch.isfinite(out[70:].view(torch.bfloat16).float()).all()


def test_equal_calls_give_equal_bits():
    inp = ref.chunk_batch([(64, 6000), (500, 900), (1, 40)], 8, 2, 128, seed=5)
    a, za = run(inp)
    for _ in range(3):
        b, zb = run(inp)
        assert torch.equal(a, b) and torch.equal(za, zb)


def test_many_requests():
    rng = np.random.default_rng(3)
    lengths = []
    for _ in range(300):
        q = int(rng.integers(0, 12))
        lengths.append((q, q + int(rng.integers(0, 90))))
    run(ref.chunk_batch(lengths, 4, 2, 64, seed=7))
    run(ref.chunk_batch(lengths[:65], 4, 2, 128, "fp8", seed=7))


def test_single_rows_agree_with_verify_attention(oracle):
    """Chains of up to 21 new tokens: what the call for them is bound to, too."""
    from paper_2604_09562_amd import synth
    cfg = synth.CONFIGS[1].scaled(batch=9, ctx=("uniform", 21, 900), depth=("uniform", 0, 20))
    host = synth.make_attention_inputs(cfg, seed=3)
    want, lse = oracle.verify_attn(host)
    d = binding.attention_to_device(host)
    out, z, ws = binding.alloc_chunk_outputs(d)
    binding.ss_chunk_attn(d, out, z, ws)
    torch.cuda.synchronize()
    got = binding.bf16_bits_to_float(out)
    assert np.all(np.abs(got - want) <= 2e-2 + 1e-2 * np.abs(want))
    assert np.all(np.abs(z.cpu().numpy() - lse) <= 1e-3 + 1e-3 * np.abs(lse))


def test_another_stream():
    inp = ref.chunk_batch([(64, 3000), (300, 300)], 8, 2, 128, seed=5)
    want, zw = run(inp)
    out, z, ws = binding.alloc_chunk_outputs(inp)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        binding.ss_chunk_attn(inp, out, z, ws)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(z, zw)


def test_captured_and_replayed_with_other_lengths():
    """A graph for a padded batch: the lengths, rows and tables in it change from replay to replay."""
    big = ref.chunk_batch([(200, 900), (64, 3000), (1, 500), (30, 30)], 8, 2, 128, seed=5, spare_rows=20)
    out, z, ws = binding.alloc_chunk_outputs(big)
    binding.ss_chunk_attn(big, out, z, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ss_chunk_attn(big, out, z, ws)
    for lengths in ([(200, 900), (64, 3000), (1, 500), (30, 30)], [(1, 900), (300, 2500), (0, 0), (0, 0)], [(0, 5), (0, 0), (0, 1), (1, 1)]):
        q = [n for n, _ in lengths]
        big["q_indptr"].copy_(torch.tensor([0] + list(np.cumsum(q)), dtype=torch.int32))
        big["kv_len"].copy_(torch.tensor([n for _, n in lengths], dtype=torch.int32))
        for _ in range(2):
            out.fill_(0)
            graph.replay()
            torch.cuda.synchronize()
            ref.check_chunk(big, out, z, str(lengths))


def test_option_validate_names_the_request():
    binding.ss_set_option("validate", 1)
    try:
        good = ref.chunk_batch([(20, 40), (0, 0), (3, 50)], 4, 2, 64, spare_rows=4)
        run(good)
        for change, text in ((lambda d: d["kv_len"].__setitem__(2, 16 * 99), "request 2"), (lambda d: d["block_table"].__setitem__((0, 1), 77777), "block 1"),
                             (lambda d: d["q_indptr"].__setitem__(1, 30), "request 0"), (lambda d: d["q_indptr"].__setitem__(3, 99), "request 2"),
                             (lambda d: d["kv_len"].__setitem__(0, -1), "kv_len -1")):
            bad = ref.chunk_batch([(20, 40), (0, 0), (3, 50)], 4, 2, 64, spare_rows=4)
            out, z, ws = binding.alloc_chunk_outputs(bad)
            change(bad)
            with pytest.raises(binding.SpecVerifyError, match=text):
                binding.ss_chunk_attn(bad, out, z, ws)
        with pytest.raises(binding.SpecVerifyError, match="at most 19"):
            binding.ss_chunk_attn(good, *binding.alloc_chunk_outputs(good), max_q_len=19)
    finally:
        binding.ss_set_option("validate", 0)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_scales_that_are_not_finite(q, value):
    """They reach the rows that see their block and no other."""
    inp = ref.chunk_batch([(150, 200)], 4, 1, 128, "fp8", q, seed=3)
    blk = int(inp["block_table"][0, 7])                  # seen from position 112 on, row 62
    out, z, ws = binding.alloc_chunk_outputs(inp)
    binding.ss_chunk_attn(inp, out, z, ws)
    for name in ("k_scale", "v_scale"):
        odd = dict(inp, **{name: inp[name].clone()})
        odd[name][blk] = value
        got, zg, _ = binding.alloc_chunk_outputs(odd)
        binding.ss_chunk_attn(odd, got, zg, ws)
        torch.cuda.synchronize()
        assert torch.equal(got[:62], out[:62]) and torch.equal(zg[:62], z[:62])
        x = got[62:] if q == "f32" else got[62:].view(torch.bfloat16).float()
        assert not torch.isfinite(x).any(-1).any()


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_scales_far_from_one(q):
    inp = ref.chunk_batch([(70, 300), (1, 40), (33, 90)], 8, 2, 128, "fp8", q, seed=13)
    for b, (of_keys, of_values) in enumerate(((1e-33, 1e33), (1.0, 1e-33), (1e-42, 1e30))):
        ids = inp["block_table"][b, :ref.blocks(int(inp["kv_len"][b]))].long()
        inp["k_scale"][ids] *= of_keys
        inp["v_scale"][ids] *= of_values
    run(inp)


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_a_scale_of_scores_near_zero(q, kv):
    run(dict(ref.chunk_batch([(70, 300), (1, 40)], 8, 2, 64, kv, q, seed=14), sm_scale=1e-44))


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("d", [64, 128])
def test_without_lse(q, kv, d):
    """A form of its own, with whole tiles, merged ones, and rows that see nothing."""
    run(ref.chunk_batch([(200, 200), (64, 5000), (1, 1), (30, 10), (1, 700)], 8, 2, d, kv, q, seed=d + 1, spare_rows=2), lse=False)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_rows_with_one_weight(kv):
    """All weight on one key, far from the first ones: the output is its value, to the rounding of the output.

    The sum that divides is that of the weights as rounded, so the weight's own rounding (up to 2^-8) is not in the result; what is left are the other
    weights, below 2^-12 in all, and half a step of bf16.
    """
    n, d = 900, 128
    inp = ref.chunk_batch([(40, n)], 4, 1, d, kv, seed=15)
    blk, place = int(inp["block_table"][0, 500 // 16]), 500 % 16
    direction = torch.randn(d, generator=torch.Generator().manual_seed(1)).sign()
    key = (direction * 2.0).cuda()
    k = inp["k_cache"].float()
    k[:, 0] *= 0.125                                   # other scores: small
    k[blk, 0, place] = key / (inp["k_scale"][blk, 0] if kv == "fp8" else 1.0)
    inp["k_cache"] = k.clamp(-448.0, 448.0).to(inp["k_cache"].dtype)
    inp["q"] = (direction.cuda() * torch.linspace(1.1, 1.4, 40 * 4, device="cuda").view(40, 4, 1)).to(torch.bfloat16)
    out, _ = run(inp)
    value = inp["v_cache"][blk, 0, place].float() * (inp["v_scale"][blk, 0] if kv == "fp8" else 1.0)
    got = out.view(torch.bfloat16).float()
    x = (inp["q"].float() * key).sum(-1) / d ** 0.5     # its score: 24 and more
    assert float(x.min()) > 20.0
    size = ref.chunk_reference(inp)[2].float().amax(-1, keepdim=True) + value.abs().max()
    assert ((got - value).abs() <= value.abs() * 2.0 ** -8 + size * 2.0 ** -12 + n * torch.exp(-x.min() + 8.0) * 6.0).all()


@pytest.mark.parametrize("lse", [True, False])
@pytest.mark.parametrize("kv,d", [("bf16", 128), ("fp8", 128), ("bf16", 64), ("fp8", 64)])
@pytest.mark.parametrize("lengths,hq,hkv", [([(389, 489)], 32, 8), ([(385, 485)], 32, 8), ([(519, 519)], 8, 8), ([(521, 521)], 8, 8), ([(259, 259)], 16, 8), ([(1031, 1031)], 8, 8),
                                            ([(700, 1500), (300, 333), (513, 513)], 8, 4)])
def test_last_tiles_that_are_not_full(lengths, hq, hkv, kv, d, lse):
    """Requests of three tiles and more whose last one is short: what is merged is what was written (the workspace holds NaN before)."""
    run(ref.chunk_batch(lengths, hq, hkv, d, kv, seed=hq, spare_rows=2), lse=lse)


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (4, 2), (5, 1), (14, 2), (16, 1)])
def test_groupings_of_several_tiles(q, kv, hq, hkv):
    run(ref.chunk_batch([(1100, 1500), (333, 800), (1, 90), (600, 600)], hq, hkv, 64, kv, q, seed=hq))


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "fp8")])
@pytest.mark.parametrize("hq,d,chunk,n", [(4, 128, 150, 200), (2, 128, 300, 700), (2, 64, 300, 700), (16, 128, 40, 333), (2, 128, 128, 128)])
def test_values_that_are_not_finite(q, kv, hq, d, chunk, n):
    """A value that is not finite reaches its column of the rows that see it, whichever step it is in, and nothing else changes by a bit.

    Two KV heads; the last tiles leave wavefronts without rows.
    """
    inp = ref.chunk_batch([(chunk, n), (1, 40)], hq, 2, d, kv, q, seed=3)
    G = hq // 2
    want, zw = run(inp)
    bits = lambda x: x.contiguous().view(torch.uint8)  # noqa: E731
    _, _, ws = binding.alloc_chunk_outputs(inp)
    for i, pos in enumerate(sorted({0, n - chunk, n - chunk // 2} | set(range(n - 1, max(n - 140, -1), -16)))):
        blk, place = int(inp["block_table"][0, pos // 16]), pos % 16
        odd = dict(inp, v_cache=inp["v_cache"].clone())
        raw = odd["v_cache"].view(torch.uint8) if kv == "fp8" else odd["v_cache"]
        raw[blk, 0, place, 5] = (0x7F, 0xFF)[i % 2] if kv == "fp8" else (float("inf"), float("nan"), -float("inf"))[i % 3]
        got, zg, _ = binding.alloc_chunk_outputs(inp)
        ws.fill_(0xFF)
        binding.ss_chunk_attn(odd, got, zg, ws)
        torch.cuda.synchronize()
        row = max(pos - (n - chunk), 0)                  # the first one that sees it
        hit = (got if q == "f32" else got.view(torch.bfloat16))[row:chunk, :G, 5]
        assert not torch.isfinite(hit).any(), f"position {pos}: {int(torch.isfinite(hit).sum())} of {hit.numel()} rows do not have it"
        got[row:chunk, :G, 5] = want[row:chunk, :G, 5]
        assert torch.equal(bits(got), bits(want)) and torch.equal(zg, zw), f"position {pos}"


@pytest.mark.parametrize("lse", [True, False])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("q,kv,d", [("bf16", "bf16", 128), ("bf16", "fp8", 128), ("bf16", "bf16", 64), ("bf16", "fp8", 64), ("f32", "f32", 128), ("f32", "bf16", 64), ("f32", "fp8", 64)])
def test_scores_of_the_whole_fp32_range(q, kv, d, sign, lse):
    """Scores of every second head from +-1e32 to +-2e37, products to 1.6e38: the largest takes all of the weight, whatever its sign.  The other heads' are ordinary.

    One product to a score, no two the same: a score is off by three roundings at most (product, scale, factor of powers of two), the next one by 2^-7 of it or, in
    e4m3 blocks, 2^-17 by their scales.  The weight of the largest is one and the others' zero, so the output is its value, rounded once if to bf16 (the sum
    that divides is one), and the log-sum-exp the score, to the score's roundings and three more.
    """
    lengths = [(3, 3), (70, 200), (64, 1100), (1, 40), (300, 500)]
    inp = ref.chunk_batch(lengths, 8, 2, d, kv, q, seed=3)
    rng = np.random.default_rng(5)
    shape = inp["k_cache"].shape
    bits = lambda x: int(np.float32(x).view(np.uint32)) >> 16  # noqa: E731
    if kv == "fp8":                                      # codes 2^-6 .. 448 of blocks whose scales all differ
        codes = rng.integers(8, 127, shape[:3]).astype(np.uint8)
        for row in codes.reshape(-1, 16):
            row[:] = rng.choice(np.arange(8, 127), 16, replace=False)
        steps = rng.permutation(shape[0] * shape[1]).reshape(shape[:2])
        inp["k_scale"] = torch.from_numpy((sign * 10.0 ** (15.8 + 0.2 * (steps + rng.random(shape[:2]) * 0.5) / steps.size)).astype(np.float32)).cuda()
        k = torch.zeros(shape, dtype=torch.uint8)
        k[..., 5] = torch.from_numpy(codes)
        inp["k_cache"] = k.cuda().view(torch.float8_e4m3fn)
    else:                                                # every bf16 number at most once to a head
        sizes = np.stack([rng.permutation(np.arange(bits(1e14), bits(1e19)))[:shape[0] * 16] for _ in range(shape[1])], 1)
        sizes = (sizes.astype(np.uint32) << 16).view(np.float32).reshape(shape[0], 16, shape[1]).transpose(0, 2, 1)
        k = torch.zeros(shape)
        k[..., 5] = torch.from_numpy(sign * sizes.copy())
        inp["k_cache"] = k.cuda().to(inp["k_cache"].dtype)
    query = torch.zeros_like(inp["q"])
    query[:, 0::2, 5] = 1.6e19
    query[:, 1::2, 5] = 1.0e-17
    inp["q"] = query
    out, z, ws = binding.alloc_chunk_outputs(inp)
    ws.fill_(0xFF)
    binding.ss_chunk_attn(inp, out, z if lse else None, ws)
    torch.cuda.synchronize()
    got = (out if q == "f32" else out.view(torch.bfloat16)).double()
    want, zw, size, mag = ref.chunk_reference(inp)
    tol, ltol = ref.chunk_tolerances(inp, want, zw, size, mag)
    assert ((got - want).abs() <= tol)[:, 1::2].all(), "ordinary heads"
    assert not lse or ((z.double() - zw).abs() <= ltol)[:, 1::2].all()
    row = 0
    for b, (chunk, n) in enumerate(lengths):
        ids = inp["block_table"][b, :ref.blocks(n)].long()
        for h in range(2):
            part = lambda c, sc: (c.view(torch.uint8)[:, h][ids].view(c.dtype) if kv == "fp8" else c[:, h][ids]).double() * (1.0 if sc is None else sc[ids, h].double()[:, None, None])  # noqa: E731
            keys, values = part(inp["k_cache"], inp["k_scale"]).reshape(-1, d)[:n, 5], part(inp["v_cache"], inp["v_scale"]).reshape(-1, d)[:n]
            for head in (4 * h, 4 * h + 2):
                x = inp["q"][row:row + chunk, head, 5].double()[:, None] * keys * inp["sm_scale"]
                last = torch.arange(chunk, device="cuda") + n - chunk
                x = torch.where(torch.arange(n, device="cuda") <= last[:, None], x, -float("inf"))
                top, at = x.topk(min(2, n), -1)
                assert n == 1 or (top[:, 0] - top[:, 1] > top[:, 0].abs() * 2.0 ** -20)[last > 0].all()
                o = got[row:row + chunk, head]
                # (a scale of values in the chunk's bf16 form: its fraction goes through a logarithm and an exponential of about 2^-22 each)
                bound = values[at[:, 0]].abs() * ((2.0 ** -8 if q == "bf16" else 0.0) + 2.0 ** -20) + 1e-30
                assert ((o - values[at[:, 0]]).abs() <= bound).all(), f"request {b}, head {head}"
                if lse:
                    assert ((z[row:row + chunk, head].double() - top[:, 0]).abs() <= top[:, 0].abs() * 2.0 ** -21).all(), f"request {b}, head {head}"
        row += chunk


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
def test_references_that_rise_from_far_below(q, kv):
    """Scores of a row go from -1e33 at its first keys to ordinary ones, and from ordinary ones to 1e33: what came before has no weight left."""
    n, d = 800, 128
    for first, sign in ((400, -1.0), (400, 1.0)):
        inp = ref.chunk_batch([(100, n)], 4, 1, d, kv, q, seed=8, sharp=1.0)
        ids = inp["block_table"][0].long()
        k = torch.zeros(inp["k_cache"].shape, dtype=torch.float32, device="cuda")
        k[ids, 0] = torch.randn((ids.numel(), 16, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
        big = (torch.arange(ids.numel() * 16, device="cuda") < first) if sign < 0 else (torch.arange(ids.numel() * 16, device="cuda") == first)
        k[ids, 0, :, 7] = torch.where(big, sign * 1.0e15, 0.0).view(-1, 16)
        if kv == "fp8":                                  # (a block's own scale is 1e13 where it holds what is large)
            rows = ids[big.view(-1, 16).any(-1)]
            inp["k_scale"].fill_(0.05)
            inp["k_scale"][rows] = 1.0e13
            k = (k / inp["k_scale"][..., None, None]).clamp(-448.0, 448.0)
        inp["k_cache"] = k.to(inp["k_cache"].dtype)
        query = inp["q"].clone()
        query[..., 7] = 1.0e19
        inp["q"] = query
        out, z, ws = binding.alloc_chunk_outputs(inp)
        ws.fill_(0xFF)
        binding.ss_chunk_attn(inp, out, z, ws)
        torch.cuda.synchronize()
        got = (out if q == "f32" else out.view(torch.bfloat16)).double()
        if sign < 0:                                     # the rows as if the first keys were not there
            want, zw, size, mag = ref.chunk_reference(inp)
            ordinary = dict(inp, q=query.clone())
            ordinary["q"][..., 7] = 0.0                  # (the magnitudes of the scores that count)
            tol, ltol = ref.chunk_tolerances(inp, want, zw, size, ref.chunk_reference(ordinary)[3])
            assert ((got - want).abs() <= tol).all() and ((z.double() - zw).abs() <= ltol).all()
        else:
            blk, place = int(ids[first // 16]), first % 16
            value = inp["v_cache"][blk, 0, place].double() * (inp["v_scale"][blk, 0].double() if kv == "fp8" else 1.0)
            assert ((got - value).abs() <= value.abs() * ((2.0 ** -8 if q == "bf16" else 0.0) + 2.0 ** -20)).all()


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "fp8")])
def test_requests_with_impossible_lengths_or_blocks(q, kv):
    """They are left out or read what is in the cache; nothing outside the arrays is touched, and the other requests' rows are what they were."""
    lengths = [(90, 333), (130, 400), (5, 900), (200, 200)]
    inp = ref.chunk_batch(lengths, 8, 2, 128, kv, q, seed=4, spare_rows=7)
    want, zw = run(inp)
    starts = inp["q_indptr"].tolist()
    big = 2 ** 31 - 1

    def call(**change):
        d = dict(inp, **{k: inp[k].clone() for k in ("kv_len", "q_indptr", "block_table")})
        for name, (at, value) in change.items():
            d[name][at] = torch.tensor(value, dtype=torch.int32, device="cuda")
        out, z, ws = binding.alloc_chunk_outputs(d)
        out.view(torch.uint8).fill_(0x5A)
        z.fill_(123.0)
        ws.fill_(0xFF)
        binding.ss_chunk_attn(d, out, z, ws)
        torch.cuda.synchronize()
        return out, z

    bits = lambda x: x.contiguous().view(torch.uint8)  # noqa: E731

    def same(got, requests):
        for b in requests:
            rows = slice(starts[b], starts[b + 1])
            ref.check_chunk(dict(inp, batch=1, block_table=inp["block_table"][b:b + 1], kv_len=inp["kv_len"][b:b + 1], q=inp["q"][rows],
                                 q_indptr=torch.tensor([0, lengths[b][0]], dtype=torch.int32, device="cuda"), total_rows=lengths[b][0]), got[0][rows], got[1][rows])

    for ids in (-1, big, -big - 1, inp["num_blocks"]):                      # (as many steps as before: the same cuts, the same bits)
        got = call(block_table=((1, slice(3, None)), ids))
        for b in (0, 2, 3):
            rows = slice(starts[b], starts[b + 1])
            assert torch.equal(bits(got[0][rows]), bits(want[rows])) and torch.equal(got[1][rows], zw[rows])
        assert (got[0].view(torch.uint8)[starts[-1]:] == 0x5A).all() and (got[1][starts[-1]:] == 123.0).all()
    for n in (inp["max_blocks_per_seq"] * 16 + 1, big):                     # a request that is left out
        got = call(kv_len=(1, n))
        same(got, (0, 2, 3))
        left = slice(starts[1], starts[2])
        assert (got[0].view(torch.uint8)[left] == 0x5A).all() and (got[1][left] == 123.0).all()
    for end in (inp["total_rows"] + 1, big, starts[3] - 1, -3):             # the last one's rows end outside the call's, or in front of where they begin
        got = call(q_indptr=(4, end))
        same(got, (0, 1, 2))
        assert (got[0].view(torch.uint8)[starts[3]:] == 0x5A).all() and (got[1][starts[3]:] == 123.0).all()
    got = call(kv_len=(1, -big - 1))
    same(got, (0, 2, 3))
    assert (bits(got[0][starts[1]:starts[2]]) == 0).all() and torch.isinf(got[1][starts[1]:starts[2]]).all()
    out, z, ws = binding.alloc_chunk_outputs(inp)
    out.view(torch.uint8).fill_(0x5A)
    binding.ss_chunk_attn(dict(inp, num_blocks=0), out, z, ws)              # no block at all
    torch.cuda.synchronize()
    assert (out.view(torch.uint8) == 0x5A).all()
