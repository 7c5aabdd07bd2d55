"""ss_block_map against its definition with a list: every whole number equal."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding
from tests import prefill_ref as ref

pytestmark = pytest.mark.gpu


def on_gpu(c):
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    rows = c["total_rows"]
    d = dict(batch=c["table"].shape[0], max_blocks_per_seq=c["table"].shape[1], block_table=t(c["table"]), kv_len=t(c["kv_len"]),
             q_indptr=t(c["q_indptr"]), total_rows=rows, num_blocks=c["num_blocks"], free_ids=t(c["ids"]),
             free_count=torch.tensor([c["count"]], dtype=torch.int32, device="cuda"), held=t(c["held"]))
    outs = (torch.full((rows,), -77, dtype=torch.int32, device="cuda"), torch.full((rows,), -77, dtype=torch.int32, device="cuda"),
            torch.full((1,), -77, dtype=torch.int32, device="cuda"))
    return d, outs, binding.alloc_block_map_workspace(d)


def check(c, d, outs):
    torch.cuda.synchronize()
    want = ref.block_map(c["table"], c["held"], c["ids"], c["count"], c["kv_len"], c["q_indptr"], c["total_rows"], c["num_blocks"])
    got = (d["block_table"], d["held"], d["free_ids"], d["free_count"], *outs)
    names = ("table", "held", "free list", "free count", "slots", "positions", "status")
    for name, g, w in zip(names, (got[0], got[1], got[2], got[3], got[4], got[5], got[6]), want):
        assert np.array_equal(g.cpu().numpy().reshape(-1), np.asarray(w).reshape(-1)), name
    return want


def run(c, positions=True):
    d, outs, ws = on_gpu(c)
    binding.ss_block_map(d, outs[0], outs[1] if positions else None, outs[2], ws)
    if not positions:
        outs[1].copy_(torch.from_numpy(ref.block_map(c["table"], c["held"], c["ids"], c["count"], c["kv_len"], c["q_indptr"], c["total_rows"],
                                                     c["num_blocks"])[5]))
    return check(c, d, outs)


def random_batch(seed, B, q_hi, ctx_hi, leaving=0, **kw):
    rng = np.random.default_rng(seed)
    lengths, held = [], []
    for b in range(B):
        if b < leaving:
            lengths.append((0, 0))
            held.append(int(rng.integers(0, 40)))
            continue
        q = int(rng.integers(0, q_hi + 1))
        n = q + int(rng.integers(0, ctx_hi + 1))
        lengths.append((q, n))
        held.append(max(0, ref.blocks(n - q) + int(rng.integers(0, 4)) * int(rng.random() < 0.3)))
    order = rng.permutation(B)
    return ref.map_batch([lengths[i] for i in order], [held[i] for i in order], seed=seed, **kw)


@pytest.mark.parametrize("lengths,held", [
    ([(1, 1)], [0]), ([(1, 16)], [1]), ([(1, 17)], [1]), ([(16, 16)], [0]), ([(17, 40)], [2]), ([(0, 0)], [0]), ([(0, 0)], [5]),
    ([(0, 33)], [3]), ([(0, 33)], [7]), ([(5, 5), (0, 0), (3, 50)], [0, 4, 3]), ([(3, 50), (0, 0), (5, 5)], [3, 4, 0]),
    ([(0, 0), (64, 64)], [4, 0]), ([(0, 0), (65, 65)], [4, 0]), ([(0, 0), (63, 63), (0, 0)], [9, 0, 1]), ([(2, 2)] * 64, [0] * 64),
])
def test_small(lengths, held):
    want = run(ref.map_batch(lengths, held))
    assert want[-1] == 0


@pytest.mark.parametrize("seed,B,q_hi,ctx_hi,leaving", [(1, 64, 9, 4096, 0), (2, 64, 9, 300, 20), (3, 1, 5000, 0, 0), (4, 300, 40, 200, 100),
                                                        (5, 1024, 3, 100, 300), (6, 1025, 3, 100, 300), (7, 3000, 2, 60, 500), (8, 16, 2000, 4000, 3),
                                                        (9, 1025, 9, 100, 5), (10, 2500, 6, 40, 1)])
def test_batches(seed, B, q_hi, ctx_hi, leaving):
    assert run(random_batch(seed, B, q_hi, ctx_hi, leaving, spare_rows=seed % 3 * 5, spare_columns=seed % 2 * 3))[-1] == 0


@pytest.mark.parametrize("rows", [4095, 4096, 4097])
def test_both_sides_of_the_row_count_that_takes_two_launches(rows):
    run(ref.map_batch([(rows - 7, rows + 30), (3, 20), (0, 0), (4, 4)], [2, 3, 11, 0]))


def test_blocks_pass_between_requests_within_a_call():
    c = ref.map_batch([(0, 0), (32, 32)], [2, 0], extra_free=0)
    c["ids"], c["num_blocks"], c["count"] = c["ids"][:2].copy(), 2, 0
    c["table"][0, :2] = [1, 0]
    want = run(c)
    assert want[0][1, :2].tolist() == [0, 1] and want[3] == 0


@pytest.mark.parametrize("rows", [100, 6000])
def test_missing_blocks_change_nothing(rows):
    c = ref.map_batch([(rows, rows), (1, 17), (0, 0)], [0, 1, 3])
    c["count"] = 2
    d, outs, ws = on_gpu(c)
    binding.ss_block_map(d, *outs, ws)
    want = check(c, d, outs)
    assert want[-1] == ref.blocks(rows) + 1 - 3 - 2
    d["free_count"].fill_(len(c["ids"]) - 4)          # the same call with blocks enough
    c["count"] = len(c["ids"]) - 4
    binding.ss_block_map(d, *outs, ws)
    assert check(c, d, outs)[-1] == 0


@pytest.mark.parametrize("change,status", [
    (lambda c: c["kv_len"].__setitem__(1, 2), -2), (lambda c: c["kv_len"].__setitem__(2, 16 * 40), -3), (lambda c: c["held"].__setitem__(0, -1), -1),
    (lambda c: c["held"].__setitem__(0, 99), -1), (lambda c: c["q_indptr"].__setitem__(2, 1), -2), (lambda c: c["q_indptr"].__setitem__(0, 1), -1),
    (lambda c: c["q_indptr"].__setitem__(3, 50), -3), (lambda c: c.__setitem__("count", -1), -4), (lambda c: c.__setitem__("count", 10 ** 6), -4),
    (lambda c: c["kv_len"].__setitem__(0, -5), -1)])
def test_impossible_lengths_are_reported(change, status):
    c = ref.map_batch([(4, 20), (5, 5), (0, 33)], [1, 0, 3], spare_rows=2)
    change(c)
    assert run(c)[-1] == status


def test_without_positions_and_without_requests():
    run(ref.map_batch([(4, 20), (5, 5)], [1, 0]), positions=False)
    c = ref.map_batch([], [], spare_rows=9)
    c["q_indptr"] = np.zeros(1, np.int32)
    assert run(c)[-1] == 0


def test_a_lane_over_many_steps():
    """Requests come, grow, lose rejected drafts and leave; the state stays on the GPU and no block is ever held twice."""
    rng = np.random.default_rng(11)
    B, width, total = 24, 40, 500
    c = dict(table=np.full((B, width), -5, np.int32), held=np.zeros(B, np.int32), ids=rng.permutation(total).astype(np.int32), count=total,
             num_blocks=total)
    n = np.zeros(B, np.int64)
    c["kv_len"], c["q_indptr"], c["total_rows"] = n.astype(np.int32), np.zeros(B + 1, np.int32), 600
    d, outs, ws = on_gpu(c)
    for step in range(40):
        q = np.zeros(B, np.int64)
        for b in range(B):
            u = rng.random()
            if n[b] == 0:
                q[b] = rng.integers(1, 100) if u < 0.3 else 0
            elif u < 0.1:
                n[b] = 0
            else:
                n[b] = max(1, n[b] - rng.integers(0, 6))      # drafts that were not accepted
                q[b] = min(rng.integers(1, 22), width * 16 - n[b])
        while q.sum() > 600:
            q[int(q.argmax())] //= 2
        n += q
        c["kv_len"] = n.astype(np.int32)
        c["q_indptr"] = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
        d["kv_len"].copy_(torch.from_numpy(c["kv_len"]))
        d["q_indptr"].copy_(torch.from_numpy(c["q_indptr"]))
        binding.ss_block_map(d, *outs, ws)
        c["table"], c["held"], c["ids"], c["count"], slots, _, status = check(c, d, outs)
        if status:          # too many at once: the largest chunk is taken back
            n -= q
            n[int(n.argmax())] = 0
            continue
        used = [int(x) for b in range(B) for x in c["table"][b, :c["held"][b]]] + c["ids"][:c["count"]].tolist()
        assert sorted(used) == list(range(total))


def test_captured_and_replayed():
    c = random_batch(21, 64, 9, 300, 10)
    d, outs, ws = on_gpu(c)
    state = [d["block_table"], d["held"], d["free_ids"], d["free_count"]]
    saved = [x.clone() for x in state]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        binding.ss_block_map(d, *outs, ws)
        for x, y in zip(state, saved):
            x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ss_block_map(d, *outs, ws)
    for _ in range(3):
        for x, y in zip(state, saved):
            x.copy_(y)
        for x in outs:
            x.fill_(-3)
        graph.replay()
        check(c, d, outs)


@pytest.mark.parametrize("rows", [0, 9, 5000])
def test_no_requests_and_no_arrays_of_theirs(rows):
    c = ref.map_batch([], [], spare_rows=rows)
    c["q_indptr"] = np.zeros(1, np.int32)
    d, outs, ws = on_gpu(c)
    for name in ("q_indptr", "kv_len", "held", "block_table"):
        d[name] = torch.empty(0, dtype=torch.int32, device="cuda")
    assert d["q_indptr"].data_ptr() == 0
    binding.ss_block_map(d, outs[0], outs[1], outs[2], ws)
    torch.cuda.synchronize()
    assert int(outs[2]) == 0 and (outs[0] == -1).all() and (outs[1] == -1).all() and int(d["free_count"]) == c["count"]


@pytest.mark.parametrize("rows", [12, 5000])
def test_a_free_list_longer_than_the_cache(rows):
    """Also where the step takes what is too much of it."""
    c = ref.map_batch([(12, 40), (rows - 12, rows)], [0, 0])
    d, outs, ws = on_gpu(c)
    d["free_count"].fill_(c["num_blocks"] + 2)
    before = [t.clone() for t in (d["block_table"], d["held"], d["free_ids"], d["free_count"])]
    binding.ss_block_map(d, outs[0], outs[1], outs[2], ws)
    torch.cuda.synchronize()
    assert int(outs[2]) == -3 and (outs[0] == -1).all()
    assert all(torch.equal(a, b) for a, b in zip(before, (d["block_table"], d["held"], d["free_ids"], d["free_count"])))
