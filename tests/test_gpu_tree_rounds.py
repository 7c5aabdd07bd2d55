"""ss_tree_verify in rounds, the form of calls with many rows, against the definition in 64 bits.  That the sizes of SHAPES take it is asserted where the rule is compiled
for the host (test_verify_rule.py), so that these stay cases of the rounds; small calls take it where the workspace has room for no more than rounds."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .prefill_ref import DEV
from .test_gpu_tree_verify import batch, check, device

pytestmark = pytest.mark.gpu

# name: (nodes of each request, vocabulary, max_depth of the call)
SHAPES = {
    "small trees": ([3] * 200, 40000, 1),
    "two deep": ([9, 1, 30, 4, 60] * 8, 40016, 2),
    "three deep": ([12] * 64, 60001, 3),
    "empty ones": ([0, 7, 0, 0, 9, 1] * 40, 40000, 1),
    "several blocks to a wavefront": ([4, 3] * 64, 128256, 1),
    "more blocks than lanes": ([6, 20, 14], 600_001, 1),
    "to the bound": ([22] * 41, 128256, 0),
}


def least(h):
    """The room that rounds need."""
    return binding.lib().ss_tree_verify_workspace(h["batch"], 0, h["vocab"])


def check_small(h, max_depth=0):
    """As check, in rounds whatever the sizes; and the same bits as all rows at once."""
    d, out = device(h), {}
    for room in (least(h), 1 << 24):
        n, tokens, nodes, lp = binding.alloc_tree_verify_outputs(d, DEV)[:4]
        for x in (n, tokens, nodes, lp):
            x.fill_(-99)
        ws = torch.full((room,), 0xFF, dtype=torch.uint8, device=DEV)
        binding.ss_tree_verify(d, n, tokens, nodes, lp, ws, max_depth=max_depth)
        torch.cuda.synchronize()
        out[room] = (n, tokens, nodes, lp)
    assert all(torch.equal(a, b) for a, b in zip(out[least(h)], out[1 << 24]))
    w = ref.verify(h["exact"], h["q_indptr"], h["total_rows"], h["tree_parent"], h["node_tokens"], h["uniforms"], h["temp"], max_depth or 20)
    n, tokens, nodes, lp = [x.cpu().numpy() for x in out[least(h)]]
    assert np.array_equal(n, w[0]) and np.array_equal(tokens, w[1]) and np.array_equal(nodes, w[2])
    assert (np.abs(lp.astype(np.float64) - w[3]) <= 2.0 ** -24 * np.abs(w[3]) * 1.01 + 1e-12).all()      # (as in check)
    return w


def shaped(name, **kw):
    nodes, vocab, max_depth = SHAPES[name]
    return batch(nodes, vocab, **kw), max_depth


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", [n for n in SHAPES if n != "to the bound"])
def test_shapes(name, dtype):
    h, max_depth = shaped(name, dtype=dtype, seed=len(name), stray=1, hit=0.95)
    w = check(h, max_depth)
    assert w[0].max() == max_depth


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 2047, 2048, 2049, 8191, 8193, 16384, 32000, 128256])
def test_vocabularies(vocab, dtype):
    check_small(batch([25, 1, 40, 0, 3, 64], vocab, dtype, seed=vocab, stray=1))


@pytest.mark.parametrize("max_depth", [1, 2, 3, 4, 5, 19, 20])
def test_bounds_of_the_depth(max_depth):
    w = check_small(batch([60, 40, 100, 2], 500, seed=10, depth=40, hit=1.0), max_depth)
    assert w[0].max() == max_depth or max_depth > 10


@pytest.mark.parametrize("nodes,vocab", [([5] * 300, 1000), ([300, 600, 257], 9000), ([3] * 1500, 40), ([1] * 1300, 9000)])
def test_many_requests_and_large_trees(nodes, vocab):
    """More requests than a round has workgroups, and more nodes than a workgroup has lanes."""
    check_small(batch(nodes, vocab, seed=18, depth=12))


def test_several_children_with_one_token_and_parents_that_are_none():
    h = batch([8, 8], 50, seed=17)
    for b in range(2):
        r0 = h["q_indptr"][b]
        y = ref.draw(h["exact"][r0], h["temp"][b], h["uniforms"][r0])[0]
        h["tree_parent"][r0:r0 + 8] = [5, 1, -1, 0, 0, 9, 6, -2 ** 31] if b else [-1, 0, 0, 0, 2, 2, 3, 3]
        h["node_tokens"][r0:r0 + 8] = y
    w = check_small(h)
    assert w[2][0, 0] == 1 and w[2][1, 0] == 3


def test_chains_to_the_bound_of_the_depth():
    """Requests end at every depth: chains in which every token up to a place is the one that is drawn."""
    h, _ = shaped("to the bound", seed=3, hit=0.0)
    depth = [min(b, 21) for b in range(41)]
    for b in range(41):
        r0, r1 = h["q_indptr"][b:b + 2]
        h["tree_parent"][r0:r1] = np.arange(-1, r1 - r0 - 1)
        for i in range(min(depth[b], r1 - r0 - 1)):
            h["node_tokens"][r0 + i + 1] = ref.draw(h["exact"][r0 + i], h["temp"][b], h["uniforms"][r0 + i])[0]
        if depth[b] < 21:
            y = ref.draw(h["exact"][r0 + depth[b]], h["temp"][b], h["uniforms"][r0 + depth[b]])[0]
            h["node_tokens"][r0 + depth[b] + 1] = (y + 1) % h["vocab"]
    w = check(h)
    assert w[0].tolist() == [min(d, 20) for d in depth]


@pytest.mark.parametrize("temperature", [0.0, 1e-30, 0.3, 2.0, 1e30, -1.0, float("nan"), float("inf"), [0.0, 1.0, 0.7, float("inf"), 3.0, -2.0, 0.01, float("nan")] * 25])
def test_temperatures(temperature):
    h, max_depth = shaped("small trees", temperature=temperature, seed=5)
    check(h, max_depth)
    if not isinstance(temperature, list):
        check(dict(h, logits=h["logits"].float(), logit_dtype="f32"), max_depth, scalar=temperature >= 0)


def test_requests_without_rows_rows_of_no_request_and_rows_outside_the_call():
    nodes, vocab, max_depth = SHAPES["empty ones"]
    h = batch(nodes, vocab, seed=12, spare_rows=5)
    w = check(h, max_depth)
    assert (w[1][::6] == -1).all()
    h["q_indptr"][-1] = 10 ** 6
    w = check(h, max_depth)
    assert w[0][-1] == 0 and (w[1][-1] == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_infinite_logits(dtype):
    h, max_depth = shaped("small trees", dtype=dtype, temperature=0.9, seed=14)
    x, V, inf = h["logits"], h["vocab"], float("inf")
    x[0] = -inf                       # nothing left
    x[3, 5:] = -inf                   # the first five only
    x[6, :39000] = float("nan")       # NaN is masked
    x[9, 30000] = inf
    x[9, 900] = inf
    x[12] = float("nan")
    x[15] = -inf
    x[15, 2048] = -3.0                # a single token
    x[18, 100:] = -1e30               # masses that vanish
    x[21] = 3e38                      # all alike, and large
    h["exact"] = x[:, :V].double().numpy()
    w = check(h, max_depth)
    assert w[1][0, 0] == 0 and w[1][3, 0] == 900 and w[1][4, 0] == 0 and w[1][5, 0] == 2048
    check(dict(h, temp=np.zeros(200, np.float32)), max_depth)


def test_uniforms_at_their_ends():
    h, max_depth = shaped("small trees", seed=15)
    h["uniforms"][::3] = np.float32([0.0, np.nextafter(np.float32(1), np.float32(0)), 1e-30, 1 - 2.0 ** -12])[np.arange(200) % 4]
    h["logits"][::2, :39990] = -float("inf")
    h["exact"] = h["logits"][:, :h["vocab"]].double().numpy()
    w = check(h, max_depth)
    assert w[1][0, 0] == 39990


def test_captured_and_replayed():
    h, max_depth = shaped("three deep", seed=20, hit=0.9)
    check(h, max_depth, logprobs=False)
    d = device(h)
    state = binding.alloc_tree_verify_outputs(d, DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.ss_tree_verify(d, *state, max_depth=max_depth)
    for i in range(4):
        if i == 2:
            d["uniforms"].copy_(torch.rand(d["total_rows"], device=DEV))
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in state[:4]]
        for x in state:
            x.fill_(-1)
        binding.ss_tree_verify(d, *state, max_depth=max_depth)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, state[:4]))


def test_two_calls_at_once():
    cases = [shaped("small trees", seed=21), shaped("empty ones", seed=22)]
    ds = [device(h) for h, _ in cases]
    want = [ref.verify(h["exact"], h["q_indptr"], h["total_rows"], h["tree_parent"], h["node_tokens"], h["uniforms"], h["temp"], most) for h, most in cases]
    states = [binding.alloc_tree_verify_outputs(d, DEV) for d in ds]
    for _ in range(3):
        streams = [torch.cuda.Stream() for _ in ds]
        for s, d, st, (_, most) in zip(streams, ds, states, cases):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                binding.ss_tree_verify(d, *st, max_depth=most)
        torch.cuda.synchronize()
        for w, st in zip(want, states):
            assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(st[:3], w[:3]))
