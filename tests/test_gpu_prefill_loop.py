"""The three calls that fill the cache as a worker makes them: block tables and slots, then for each layer the write and the attention of the step's chunk.

Requests come and go, prompts come in pieces beside requests that decode, and blocks pass from one request to another.  Per step: tables and slots exact, the cache's
bytes exact, attention within the bounds that follow from its roundings.  Then the calls of a verify step on the same cache, and the whole as a captured graph.
"""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding, example
from tests import prefill_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Lane:
    """A cache of some layers, its tables and its free list on the GPU, and the same as lists and plain tensors."""

    def __init__(self, slots, num_blocks, width, layers, hq, hkv, d, kv, q, seed):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)
        self.hq, self.hkv, self.d, self.kv, self.q, self.layers, self.batch = hq, hkv, d, kv, q, layers, slots
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
        self.table, self.held, self.num_blocks, self.width = i32(slots, width), i32(slots), num_blocks, width
        self.free_ids = torch.randperm(num_blocks, generator=torch.Generator().manual_seed(seed)).to(torch.int32).to(DEV)
        self.free_count = torch.full((1,), num_blocks, dtype=torch.int32, device=DEV)
        self.status, self.ws = i32(1), None
        junk = lambda: ref.cache_values((num_blocks, hkv, 16, d), kv, self.gen)  # noqa: E731
        self.caches = [junk() + junk() for _ in range(layers)]       # k, k scales, v, v scales
        self.plain = [[None if t is None else t.cpu() for t in c] for c in self.caches]
        self.mirror = dict(table=self.table.cpu().numpy().copy(), held=self.held.cpu().numpy().copy(), ids=self.free_ids.cpu().numpy().copy(), count=num_blocks)

    def batch_of(self, lengths, spare=3):
        """The batch for (new tokens, length) of each slot; projections are parts of one wider row, as a worker's product gives them."""
        indptr = np.zeros(len(lengths) + 1, dtype=np.int32)
        indptr[1:] = np.cumsum([q for q, _ in lengths])
        rows = int(indptr[-1]) + spare
        d = dict(batch=self.batch, num_q_heads=self.hq, num_kv_heads=self.hkv, head_dim=self.d, block_size=16, num_blocks=self.num_blocks,
                 max_blocks_per_seq=self.width, total_rows=rows, kv_dtype=self.kv, q_dtype=self.q, new_dtype=self.q, sm_scale=1.0 / self.d ** 0.5,
                 block_table=self.table, held=self.held, free_ids=self.free_ids, free_count=self.free_count,
                 kv_len=torch.tensor([n for _, n in lengths], dtype=torch.int32, device=DEV), q_indptr=torch.from_numpy(indptr).to(DEV))
        wide = [torch.randn((rows, (self.hq + 2 * self.hkv) * self.d), generator=self.gen, device=DEV).to(ref.TORCH[self.q]) for _ in range(self.layers)]
        return d, wide, torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV)

    def layer(self, d, wide, n):
        k, ks, v, vs = self.caches[n]
        a, b = self.hq * self.d, (self.hq + self.hkv) * self.d
        return dict(d, k_cache=k, v_cache=v, k_scale=ks, v_scale=vs, q=wide[n][:, :a].unflatten(1, (self.hq, self.d)),
                    k_new=wide[n][:, a:b].unflatten(1, (self.hkv, self.d)), v_new=wide[n][:, b:].unflatten(1, (self.hkv, self.d)))

    def enqueue(self, d, wide, slot_map, positions, outs):
        self.ws = binding.alloc_block_map_workspace(d) if self.ws is None else self.ws
        binding.ss_block_map(d, slot_map, positions, self.status, self.ws)
        for n in range(self.layers):
            part = self.layer(d, wide, n)
            binding.ss_kv_write(part, slot_map)
            binding.ss_chunk_attn(part, outs[n][0], outs[n][1], outs[0][2])      # (one workspace for all layers)

    def check(self, d, wide, slot_map, positions, outs, label):
        m = self.mirror
        want = ref.block_map(m["table"], m["held"], m["ids"], m["count"], d["kv_len"].cpu().numpy(), d["q_indptr"].cpu().numpy(), d["total_rows"], self.num_blocks)
        got = (self.table, self.held, self.free_ids, self.free_count, slot_map, positions, self.status)
        for name, g, w in zip(("table", "held", "free list", "free count", "slots", "positions", "status"), got, want):
            assert np.array_equal(g.cpu().numpy().reshape(-1), np.asarray(w).reshape(-1)), f"{label}: {name}"
        m["table"], m["held"], m["ids"], m["count"] = [np.array(w) for w in want[:3]] + [int(np.asarray(want[3]).reshape(-1)[0])]
        slots = slot_map.cpu()
        for n in range(self.layers):
            part = self.layer(d, wide, n)
            for cache, scale, new in ((0, 1, part["k_new"]), (2, 3, part["v_new"])):
                self.write(self.plain[n][cache], self.plain[n][scale], new.cpu(), slots)
            for i, name in enumerate(("k", "k scales", "v", "v scales")):
                if self.caches[n][i] is not None:
                    a, b = self.caches[n][i].cpu().contiguous().view(torch.uint8), self.plain[n][i].contiguous().view(torch.uint8)
                    assert torch.equal(a, b), f"{label}: layer {n}, {name}"
            ref.check_chunk(part, outs[n][0], outs[n][1], f"{label}, layer {n}")

    @staticmethod
    def write(cache, scale, new, slots):
        rows = (slots >= 0).nonzero()[:, 0]
        blk, place = slots[rows].long() // 16, slots[rows].long() % 16
        if scale is None:
            cache[blk, :, place] = new[rows].to(cache.dtype)
            return
        x = new[rows].float()
        for b in blk.unique().tolist():
            here = blk == b
            if (place[here] == 0).any():
                top = x[here].abs().amax((0, 2)) / torch.tensor(448.0)
                scale[b] = torch.where(top > 0, top, torch.ones(()))
        code = (x / scale[blk][..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        cache.view(torch.uint8)[blk, :, place] = code.view(torch.uint8)


# per step: (new tokens, length after the step) of each of the five slots
STEPS = [
    [(200, 200), (37, 37), (0, 0), (0, 0), (0, 0)],                  # two prompts come, one of them its first 200 tokens
    [(256, 456), (1, 38), (16, 16), (0, 0), (500, 500)],             # its next piece beside a request that decodes
    [(31, 487), (5, 43), (17, 33), (0, 0), (0, 500)],                # the last piece; drafts; a request that waits
    [(1, 488), (2, 42), (300, 333), (64, 64), (0, 0)],               # drafts taken back; a request leaves
    [(0, 0), (8, 50), (1, 334), (1, 65), (450, 450)],                # another leaves, a new one takes its blocks
]


@pytest.mark.parametrize("kv,q,hq,hkv,d", [("bf16", "bf16", 8, 2, 128), ("fp8", "bf16", 8, 2, 128), ("f32", "f32", 4, 1, 64), ("fp8", "f32", 6, 2, 64)])
def test_prompts_in_pieces_beside_decoding(kv, q, hq, hkv, d):
    lane = Lane(5, 80, 33, 2, hq, hkv, d, kv, q, seed=hq + d)
    for i, lengths in enumerate(STEPS):
        b, wide, slot_map, positions = lane.batch_of(lengths)
        outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0)) for _ in range(2)]
        lane.enqueue(b, wide, slot_map, positions, outs)
        torch.cuda.synchronize()
        lane.check(b, wide, slot_map, positions, outs, f"step {i}")


def test_a_step_that_lacks_blocks_writes_nothing():
    lane = Lane(2, 10, 33, 1, 4, 2, 64, "bf16", "bf16", seed=1)
    for lengths in ([(100, 100), (40, 40)], [(90, 190), (1, 41)], [(1, 101), (8, 48)]):   # 7 + 3 blocks; 12 + 3; 7 + 3
        b, wide, slot_map, positions = lane.batch_of(lengths)
        before = [t.clone() for t in (lane.caches[0][0], lane.caches[0][2], lane.table, lane.held)]
        outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0))]
        binding.ss_block_map(b, slot_map, positions, lane.status, binding.alloc_block_map_workspace(b))
        part = lane.layer(b, wide, 0)
        binding.ss_kv_write(part, slot_map)
        torch.cuda.synchronize()
        if lengths[0][1] == 190:
            assert int(lane.status) == 5 and (slot_map == -1).all()
            assert all(torch.equal(x, y) for x, y in zip(before, (lane.caches[0][0], lane.caches[0][2], lane.table, lane.held)))
            continue
        assert int(lane.status) == 0
        binding.ss_chunk_attn(part, *outs[0])
        torch.cuda.synchronize()
        lane.check(b, wide, slot_map, positions, outs, str(lengths))


def test_the_verify_step_reads_what_was_filled():
    """Drafts behind a prompt: the two attention calls of the library on the same cache, each within its own bound of the other."""
    lane = Lane(3, 80, 33, 1, 8, 2, 128, "bf16", "bf16", seed=5)
    for lengths in ([(400, 400), (33, 33), (150, 150)], [(4, 404), (1, 34), (7, 157)]):
        b, wide, slot_map, positions = lane.batch_of(lengths, spare=0)
        outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0))]
        lane.enqueue(b, wide, slot_map, positions, outs)
    part = lane.layer(b, wide, 0)
    part["q"] = part["q"].contiguous().view(torch.int16)
    out, lse, ws = binding.alloc_attention_outputs(part, max_q_len=7)
    binding.ss_spec_verify_attn(part, out, lse, ws, max_q_len=7)
    torch.cuda.synchronize()
    part["q"] = lane.layer(b, wide, 0)["q"]
    want = ref.chunk_reference(part)
    tol, ltol = ref.chunk_tolerances(part, *want)
    for o, z in ((out, lse), outs[0][:2]):
        assert ((o.view(torch.bfloat16).double() - want[0]).abs() <= tol).all() and ((z.double() - want[1]).abs() <= ltol).all()


@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_captured_steps(kv, q):
    """One step recorded on a stream of its own: every replay from the same state gives the eager call's bits, with eager work on the same workspaces between."""
    lane = Lane(5, 80, 33, 2, 8, 2, 128, kv, q, seed=9)
    b, wide, slot_map, positions = lane.batch_of(STEPS[0])
    outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0)) for _ in range(2)]
    lane.enqueue(b, wide, slot_map, positions, outs)
    b, wide, slot_map, positions = lane.batch_of(STEPS[1])
    outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0)) for _ in range(2)]
    state = [lane.table, lane.held, lane.free_ids, lane.free_count] + [t for c in lane.caches for t in c if t is not None]
    torch.cuda.synchronize()
    saved = [t.clone() for t in state]

    def restore():
        for t, s in zip(state, saved):
            t.copy_(s)
        for o in outs:
            o[0].view(torch.uint8).fill_(0x33)
            o[1].fill_(5.0)
        outs[0][2].fill_(0xFF)
        lane.ws.fill_(0xFF)
        slot_map.fill_(-9)
        torch.cuda.synchronize()

    restore()
    lane.enqueue(b, wide, slot_map, positions, outs)
    torch.cuda.synchronize()
    results = state + [slot_map, positions, lane.status] + [t for o in outs for t in o[:2]]
    want = [t.clone() for t in results]
    restore()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        lane.enqueue(b, wide, slot_map, positions, outs)             # warm-up on the capture stream
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            lane.enqueue(b, wide, slot_map, positions, outs)
    torch.cuda.synchronize()
    for replay in range(4):
        restore()
        graph.replay()
        torch.cuda.synchronize()
        for i, (t, w) in enumerate(zip(results, want)):
            assert torch.equal(t.contiguous().view(torch.uint8), w.contiguous().view(torch.uint8)), f"replay {replay}: result {i}"


@pytest.mark.parametrize("chunk", [64, 2000])
def test_the_example_with_prompts_in_chunks(chunk):
    r = example.run(steps=2, batch=4, layers=2, vocab=4096, seed=1, verbose=False, chunk=chunk)
    assert int((r["kv_len"] - r["start_len"]).sum()) == r["emitted"]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_blocks_behind_four_gigabytes(kv):
    """Offsets into a long cache pass 32 bits: blocks at its end, written and attended."""
    num_blocks, hkv, d = 300000, 8, 128
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    lengths = [(70, 70), (20, 20)]
    ids = torch.arange(num_blocks - 8, num_blocks, dtype=torch.int32, device=DEV).flip(0)
    table = torch.zeros((2, 5), dtype=torch.int32, device=DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    free = torch.empty(num_blocks, dtype=torch.int32, device=DEV)
    free[:8] = ids
    b = dict(batch=2, num_q_heads=16, num_kv_heads=hkv, head_dim=d, block_size=16, num_blocks=num_blocks, max_blocks_per_seq=5, total_rows=90, kv_dtype=kv,
             q_dtype="bf16", new_dtype="bf16", sm_scale=d ** -0.5, block_table=table, held=i32([0, 0]), free_ids=free, free_count=i32([8]), kv_len=i32([70, 20]),
             q_indptr=i32([0, 70, 90]))
    for name in ("k", "v"):
        b[name + "_cache"] = torch.empty((num_blocks, hkv, 16, d), dtype=ref.TORCH[kv], device=DEV)
        b[name + "_scale"] = torch.empty((num_blocks, hkv), device=DEV) if kv == "fp8" else None
        b[name + "_new"] = torch.randn((90, hkv, d), generator=gen, device=DEV).to(torch.bfloat16)
    assert b["k_cache"].nbytes > 4 << 30
    b["q"] = torch.randn((90, 16, d), generator=gen, device=DEV).to(torch.bfloat16)
    slots, status = torch.empty(90, dtype=torch.int32, device=DEV), i32([1])
    binding.ss_block_map(b, slots, None, status, binding.alloc_block_map_workspace(b))
    binding.ss_kv_write(b, slots)
    out, lse, ws = binding.alloc_chunk_outputs(b)
    binding.ss_chunk_attn(b, out, lse, ws)
    torch.cuda.synchronize()
    assert int(status) == 0 and int(slots.min()) >= 16 * (num_blocks - 8)
    place = slots.long()
    for name in ("k", "v"):
        got = b[name + "_cache"].view(torch.uint8) if kv == "fp8" else b[name + "_cache"]
        got = got[place // 16, :, place % 16]
        new = b[name + "_new"]
        if kv == "fp8":
            new = (new.float() / b[name + "_scale"][place // 16][..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(got, new)
    ref.check_chunk(b, out, lse, kv)


def test_two_workers_at_once():
    """Two batches with caches, pools and workspaces of their own on two streams give what each gives alone."""
    lanes = [Lane(5, 80, 33, 1, 8, 2, 128, "bf16", "bf16", seed=21 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in lanes]
    work = []
    for lane, lengths in zip(lanes, (STEPS[0], STEPS[0][::-1])):
        b, wide, slot_map, positions = lane.batch_of(lengths)
        work.append((b, wide, slot_map, positions, [binding.alloc_chunk_outputs(lane.layer(b, wide, 0))]))
        lane.ws = binding.alloc_block_map_workspace(b)
    torch.cuda.synchronize()
    for lane, w, stream in zip(lanes, work, streams):
        with torch.cuda.stream(stream):
            lane.enqueue(*w)
    torch.cuda.synchronize()
    for lane, w in zip(lanes, work):
        lane.check(*w, "two at once")


@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("fp8", "bf16"), ("f32", "f32")])
def test_the_whole_of_a_step_that_lacks_blocks(kv, q):
    """All three calls are enqueued before anyone knows the status: the cache stays as it was, and the step is made again."""
    lane = Lane(2, 10, 33, 1, 4, 2, 64, kv, q, seed=1)
    lane.table.fill_(-7)
    lane.mirror["table"][:] = -7
    steps = [[(100, 100), (40, 40)], [(300, 400), (1, 41)], [(20, 120), (1, 41)]]     # 7 + 3 blocks; 25 + 3; 8 + 3: one is missing; then a request leaves
    for i, lengths in enumerate(steps + [[(20, 120), (0, 0)]]):
        b, wide, slot_map, positions = lane.batch_of(lengths)
        outs = [binding.alloc_chunk_outputs(lane.layer(b, wide, 0))]
        before = [t.clone() for t in lane.caches[0] if t is not None] + [lane.table.clone(), lane.held.clone()]
        lane.enqueue(b, wide, slot_map, positions, outs)
        torch.cuda.synchronize()
        if i in (1, 2):
            assert int(lane.status) == (18, 1)[i - 1] and (slot_map == -1).all()
            after = [t for t in lane.caches[0] if t is not None] + [lane.table, lane.held]
            assert all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(before, after))
            continue
        lane.check(b, wide, slot_map, positions, outs, str(lengths))


def test_the_example_stops_where_blocks_are_missing(monkeypatch):
    """Nothing that follows the table is enqueued behind a block map that has not been made."""
    real, calls, steps = binding.ss_block_map, [], [0]

    def lacking(d, slots, positions, status, ws):
        real(d, slots, positions, status, ws)
        steps[0] += 1
        if steps[0] == 2:                                # (the prompts in one chunk, then the first decode step)
            status.fill_(4)

    monkeypatch.setattr(binding, "ss_block_map", lacking)
    for name in ("ss_kv_append", "ss_spec_verify_attn"):
        monkeypatch.setattr(binding, name, lambda *a, **k: calls.append(1))
    with pytest.raises(RuntimeError, match="status 4"):
        example.run(steps=2, batch=4, layers=1, vocab=4096, seed=1, verbose=False, chunk=4000)
    assert steps[0] == 2 and not calls


def test_tensors_that_are_not_what_a_call_writes():
    """On the GPU, where only the type, the length or the strides are wrong: refused before anything is enqueued."""
    lane = Lane(2, 10, 33, 1, 4, 2, 64, "bf16", "bf16", seed=1)
    b, wide, slots, positions = lane.batch_of([(20, 20), (5, 5)])
    d, ws = lane.layer(b, wide, 0), binding.alloc_block_map_workspace(b)
    out, z, wc = binding.alloc_chunk_outputs(d)
    n = slots.numel()
    for call, text in [
        (lambda: binding.ss_block_map(d, slots.long(), positions, lane.status, ws), "slot_map"), (lambda: binding.ss_block_map(d, slots, positions[:-1], lane.status, ws), "positions"),
        (lambda: binding.ss_block_map(d, slots, None, lane.status.float(), ws), "status"), (lambda: binding.ss_kv_write(d, slots.long()), "slot_map"),
        (lambda: binding.ss_kv_write(d, torch.zeros(2 * n, dtype=torch.int32, device=DEV)[::2]), "slot_map"), (lambda: binding.ss_kv_write(dict(d, k_new=d["k_new"].float()), slots), "k_new"),
        (lambda: binding.ss_kv_write(dict(d, v_new=d["v_new"].float()), slots), "v_new"), (lambda: binding.ss_chunk_attn(d, out.float(), z, wc), "out"),
        (lambda: binding.ss_chunk_attn(d, torch.zeros((n, 4, 128), dtype=torch.int16, device=DEV)[..., :64], z, wc), "out"), (lambda: binding.ss_chunk_attn(d, out, z.half(), wc), "lse"),
        (lambda: binding.ss_chunk_attn(d, out, z[:-1], wc), "lse"), (lambda: binding.alloc_chunk_outputs(dict(d, k_cache=d["k_cache"].float())), "k_cache"),
        (lambda: binding.alloc_chunk_outputs(dict(d, v_cache=d["v_cache"][1:])), "v_cache"), (lambda: binding.alloc_chunk_outputs(dict(d, kv_len=d["kv_len"].long())), "kv_len"),
        (lambda: binding.alloc_block_map_workspace(dict(d, held=d["held"].long())), "held"), (lambda: binding.alloc_block_map_workspace(dict(d, free_ids=d["free_ids"][1:])), "free_ids")]:
        with pytest.raises(binding.SpecVerifyError, match=text):
            call()
    binding.ss_block_map(d, slots, positions, lane.status, ws)
    torch.cuda.synchronize()
    assert int(lane.status) == 0
