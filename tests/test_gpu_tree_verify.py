"""ss_tree_verify against the definition in 64 bits: tokens, nodes and lengths equal, log-probabilities within a rounding."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .prefill_ref import DEV

pytestmark = pytest.mark.gpu


def batch(nodes, vocab, dtype="bf16", temperature=0.8, seed=0, depth=8, stray=0, spare_rows=0, spread=2.5, hit=0.8):
    """Trees whose children carry likely tokens; with probability `hit` one child of a node carries the token that the target draws there."""
    rng = np.random.default_rng(seed)
    B, R = len(nodes), sum(nodes) + spare_rows
    indptr = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    stride = (vocab + 7) // 8 * 8 + 8 * stray
    x = torch.from_numpy(rng.standard_normal((R, stride)).astype(np.float32) * spread)
    x[:, ::7] += 3.0
    logits = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    exact = logits[:, :vocab].double().numpy()
    u = rng.random(R).astype(np.float32)
    u[u >= 1.0] = 0.5
    temp = np.broadcast_to(np.asarray(temperature, np.float32), (B,)).copy()
    parent, tokens = np.full(R, -7, np.int32), rng.integers(0, vocab, R).astype(np.int32)
    for b, n in enumerate(nodes):
        r0 = indptr[b]
        parent[r0:r0 + n] = ref.random_tree(n, rng, depth)
        for i in range(n):
            below = [c for c in range(i + 1, n) if parent[r0 + c] == i]
            if below and rng.random() < hit:
                tokens[r0 + rng.choice(below)] = ref.draw(exact[r0 + i], temp[b], u[r0 + i])[0]
    return dict(batch=B, vocab=vocab, row_stride=stride, logit_dtype=dtype, total_rows=R, q_indptr=indptr, tree_parent=parent, node_tokens=tokens, logits=logits,
                uniforms=u, temp=temp, exact=exact)


def device(h, scalar=False):
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    return dict(h, q_indptr=t(h["q_indptr"]), tree_parent=t(h["tree_parent"]), node_tokens=t(h["node_tokens"]), target_logits=h["logits"].to(DEV),
                uniforms=t(h["uniforms"]), temperature=None if scalar else t(h["temp"]), temperature_scalar=float(h["temp"][0]) if len(h["temp"]) else 1.0)


def check(h, max_depth=0, scalar=False, logprobs=True):
    d = device(h, scalar)
    n, out, nodes, lp, ws = binding.alloc_tree_verify_outputs(d, DEV)
    for x in (n, out, nodes):
        x.fill_(-99)
    lp.fill_(99)
    ws.fill_(0xFF)
    binding.ss_tree_verify(d, n, out, nodes, lp if logprobs else None, ws, max_depth=max_depth)
    torch.cuda.synchronize()
    w = ref.verify(h["exact"], h["q_indptr"], h["total_rows"], h["tree_parent"], h["node_tokens"], h["uniforms"], h["temp"], max_depth or 20)
    assert np.array_equal(n.cpu().numpy(), w[0])
    assert np.array_equal(out.cpu().numpy(), w[1])
    assert np.array_equal(nodes.cpu().numpy(), w[2])
    if logprobs:
        # one rounding to 32 bits; of sums and exponentials 1e-13 and less of arguments that stay below 1e3 beside the masses that count
        off = np.abs(lp.cpu().numpy().astype(np.float64) - w[3])
        assert (off <= 2.0 ** -24 * np.abs(w[3]) * 1.01 + 1e-12).all(), off.max()
    else:
        assert (lp == 99).all()
    return w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 2047, 2048, 2049, 5000, 32000, 128256])
def test_vocabularies(vocab, dtype):
    w = check(batch([25, 1, 40, 3, 64], vocab, dtype, seed=vocab, stray=1))
    assert vocab < 100 or w[0].max() > 0


def test_a_vocabulary_of_more_blocks_than_lanes():
    check(batch([6, 2], 600_001, "bf16", seed=3))


@pytest.mark.parametrize("temperature", [0.0, 1e-30, 1e-3, 0.3, 1.0, 2.0, 50.0, 1e30, -1.0, float("nan")])
def test_temperatures(temperature):
    check(batch([25, 40, 3], 3000, "f32", temperature, seed=5))
    check(batch([25, 40, 3], 3000, "bf16", temperature, seed=6))


@pytest.mark.parametrize("nodes", [[12, 20, 1], [24] * 40])
def test_infinite_temperatures(nodes):
    """Every token alike."""
    h = batch(nodes, 5003, temperature=float("inf"), seed=16)
    check(h)
    check(h, scalar=True)


def test_a_temperature_for_each_request_or_one_for_all():
    check(batch([20] * 6, 4000, temperature=[0.0, 1.0, 0.7, 0.0, 3.0, 0.01], seed=7))
    check(batch([20] * 6, 4000, temperature=0.7, seed=8), scalar=True)
    check(batch([20] * 6, 4000, temperature=0.0, seed=9), scalar=True)


@pytest.mark.parametrize("max_depth", [1, 2, 3, 20])
def test_bound_of_the_depth(max_depth):
    h = batch([60, 40, 100], 500, seed=10, depth=40, hit=1.0)
    w = check(h, max_depth)
    assert w[0].max() == max_depth or max_depth == 20


def test_chains_deeper_than_the_row_of_nodes():
    h = batch([50, 22, 21, 20], 300, seed=11)
    for b in range(4):      # chains in which every token is the one that is drawn
        r0, r1 = h["q_indptr"][b:b + 2]
        h["tree_parent"][r0:r1] = np.arange(-1, r1 - r0 - 1)
        for r in range(r0, r1 - 1):
            h["node_tokens"][r + 1] = ref.draw(h["exact"][r], h["temp"][b], h["uniforms"][r])[0]
    w = check(h)
    assert w[0].tolist() == [20, 20, 20, 19]


def test_requests_without_rows_and_rows_of_no_request():
    w = check(batch([0, 12, 0, 0, 5, 0], 700, seed=12, spare_rows=4))
    assert (w[1][[0, 2, 3, 5]] == -1).all()
    check(batch([0, 0], 700, seed=12))


def test_rows_outside_the_call():
    h = batch([10, 12, 5], 700, seed=13)
    h["q_indptr"][3] = 10 ** 6
    w = check(h)
    assert w[0][2] == 0 and (w[1][2] == -1).all()


def test_masked_and_infinite_logits():
    h = batch([9] * 8, 2500, "f32", 0.9, seed=14)
    x = h["logits"]
    inf = float("inf")
    x[0] = -inf                       # nothing left
    x[9, 5:] = -inf                   # the first five only
    x[18, :2400] = float("nan")       # NaN is masked
    x[27, 1700] = inf
    x[27, 900] = inf
    x[36] = float("nan")
    x[45] = -inf
    x[45, 2048] = -3.0                # a single token
    x[54, 100:] = -1e30               # masses that vanish
    x[63] = 3e38                      # all alike, and large
    h["exact"] = x[:, :2500].double().numpy()
    w = check(h)
    assert w[1][0, 0] == 0 and w[1][3, 0] == 900 and w[1][4, 0] == 0 and w[1][5, 0] == 2048
    check(dict(h, temp=np.zeros(8, np.float32)))


def test_uniforms_at_their_ends():
    h = batch([1] * 6, 4100, seed=15)
    h["uniforms"][:] = [0.0, np.nextafter(np.float32(1), np.float32(0)), 0.5, 1e-30, 0.0, 1 - 2.0 ** -12]
    h["logits"][4, :4000] = -float("inf")
    h["exact"] = h["logits"][:, :4100].double().numpy()
    w = check(h)
    assert w[1][0, 0] == 0 and w[1][4, 0] == 4000


def test_equal_logits_draw_by_place():
    """All tokens alike: the token is the uniform's place, to the last one."""
    V = 4096
    h = batch([1] * 64, V, "bf16", 1.0, seed=16)
    h["logits"][:, :V] = 1.5
    h["exact"] = h["logits"][:, :V].double().numpy()
    h["uniforms"][:] = (np.arange(64) * 64 + 0.5) / V
    w = check(h)
    assert w[1][:, 0].tolist() == list(range(0, V, 64))


def test_several_children_with_one_token_and_parents_that_are_none():
    h = batch([8, 8], 50, seed=17)
    for b in range(2):
        r0 = h["q_indptr"][b]
        y = ref.draw(h["exact"][r0], h["temp"][b], h["uniforms"][r0])[0]
        h["tree_parent"][r0:r0 + 8] = [5, 1, -1, 0, 0, 9, 6, -2 ** 31] if b else [-1, 0, 0, 0, 2, 2, 3, 3]
        h["node_tokens"][r0:r0 + 8] = y
    w = check(h)
    assert w[2][0, 0] == 1 and w[2][1, 0] == 3


def test_many_requests():
    check(batch([5] * 300, 1000, seed=18))


@pytest.mark.parametrize("total", [1, 40, 600])
def test_large_trees(total):
    check(batch([total, 300], 9000, seed=19, depth=12))


def test_same_bits_again_without_log_probabilities_and_captured():
    h = batch([30, 64, 7], 32000, seed=20)
    check(h, logprobs=False)
    d = device(h)
    first = None
    state = binding.alloc_tree_verify_outputs(d, DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.ss_tree_verify(d, *state, max_depth=8)
    for i in range(3):
        if i == 2:
            d["uniforms"].copy_(torch.rand(d["total_rows"], device=DEV))
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in state[:4]]
        binding.ss_tree_verify(d, *state, max_depth=8)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, state[:4]))
        if i == 0:
            first = got
        elif i == 1:
            assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_two_calls_at_once():
    hs = [batch([30, 64, 7], 32000, seed=21), batch([25] * 20, 5000, seed=22)]
    ds = [device(h) for h in hs]
    states = [binding.alloc_tree_verify_outputs(d, DEV) for d in ds]
    for _ in range(3):
        streams = [torch.cuda.Stream() for _ in ds]
        for s, d, st in zip(streams, ds, states):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                binding.ss_tree_verify(d, *st)
        torch.cuda.synchronize()
        for h, st in zip(hs, states):
            w = ref.verify(h["exact"], h["q_indptr"], h["total_rows"], h["tree_parent"], h["node_tokens"], h["uniforms"], h["temp"], 20)
            assert np.array_equal(st[0].cpu().numpy(), w[0]) and np.array_equal(st[1].cpu().numpy(), w[1])


def test_law_of_the_first_token():
    """Whatever the tree proposes, first tokens follow the target: frequencies of 20000 draws within five standard deviations of each."""
    B, V = 20000, 12
    h = batch([3] * B, V, "f32", 1.0, seed=23)
    h["logits"][:] = h["logits"][0]
    h["uniforms"] = np.random.default_rng(24).random(3 * B).astype(np.float32)
    d = device(h)
    state = binding.alloc_tree_verify_outputs(d, DEV)
    binding.ss_tree_verify(d, *state)
    first = state[1][:, 0].cpu().numpy()
    p = np.exp(h["logits"][0, :V].double().numpy())
    p /= p.sum()
    f = np.bincount(first, minlength=V) / B
    assert (np.abs(f - p) <= 5 * np.sqrt(p * (1 - p) / B) + 1.0 / B).all()


def test_binding_refuses():
    d = device(batch([6, 6], 100, seed=25))
    state = binding.alloc_tree_verify_outputs(d, DEV)
    for name, x in (("q_indptr", d["q_indptr"].long()), ("tree_parent", d["tree_parent"][:-1]), ("node_tokens", d["node_tokens"].float()), ("uniforms", d["uniforms"].double()),
                    ("uniforms", d["uniforms"][:5]), ("temperature", d["temperature"][:1]), ("target_logits", d["target_logits"].float()),
                    ("target_logits", d["target_logits"][:-1]), ("target_logits", d["target_logits"].cpu()), ("uniforms", None)):
        with pytest.raises(binding.SpecVerifyError):
            binding.ss_tree_verify(dict(d, **{name: x}), *state)
    with pytest.raises(binding.SpecVerifyError):
        binding.ss_tree_verify(d, state[0], state[1][:1], *state[2:])
    with pytest.raises(binding.SpecVerifyError):
        binding.ss_tree_verify(d, *state[:4], state[4][:256])
