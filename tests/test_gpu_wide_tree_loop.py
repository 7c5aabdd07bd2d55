"""The calls for wide draft trees and shared blocks together, as a lane uses them: prompts, forks of them, steps with trees of any width, requests that end, a cache that is
made whole again.  After every step the cache holds exactly what each request's tokens put there."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .prefill_ref import BLOCK, DEV, TORCH, blocks

pytestmark = pytest.mark.gpu

VOCAB, HQ, HKV, D, LAYERS = 160, 8, 2, 64, 2


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Lane:
    """The books of a batch on the device, and every request's tokens on the host."""

    def __init__(self, batch, columns, num_blocks, kv, seed):
        self.rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        # what a token at a position puts into a layer's cache
        self.table = torch.randn((LAYERS, 2, VOCAB, HKV, D), device=DEV, generator=gen)
        shape = (num_blocks, HKV, BLOCK, D)
        self.layers = [dict(num_blocks=num_blocks, block_size=BLOCK, num_kv_heads=HKV, head_dim=D, kv_dtype=kv, k_scale=None, v_scale=None,
                            k_cache=torch.full(shape, float("nan"), dtype=TORCH[kv], device=DEV), v_cache=torch.full(shape, float("nan"), dtype=TORCH[kv], device=DEV)) for _ in range(LAYERS)]
        self.handle = binding.cache_layers(self.layers)
        self.kv, self.batch = kv, batch
        self.d = dict(batch=batch, max_blocks_per_seq=columns, num_blocks=num_blocks, block_table=i32(np.full((batch, columns), -1)), kv_len=i32(np.zeros(batch)),
                      held=i32(np.zeros(batch)), shares=i32(np.zeros(num_blocks)), free_ids=i32(self.rng.permutation(num_blocks)), free_count=i32([num_blocks]))
        self.status, self.ws, self.map_ws = i32([0]), binding.alloc_block_share_workspace(self.d, DEV, num_forks=batch), None
        self.tokens = [[] for _ in range(batch)]      # in the cache
        self.next = [None] * batch                    # drawn, not in the cache yet; None: no request

    def values(self, layer, side, tokens, positions):
        x = self.table[layer, side, torch.as_tensor(tokens, device=DEV)]
        return (x + torch.as_tensor(positions, device=DEV)[:, None, None] * 0.01).to(torch.bfloat16 if self.kv == "bf16" else torch.float32)

    def ok(self):
        assert int(self.status) == 0, int(self.status)

    def step_arrays(self, new):
        """Blocks and slots for new[b] tokens more of each request."""
        indptr = np.concatenate([[0], np.cumsum(new)])
        R = int(indptr[-1])
        self.d["kv_len"] += i32(new)
        self.d.update(q_indptr=i32(indptr), total_rows=R)
        slots = torch.empty(R, dtype=torch.int32, device=DEV)
        self.map_ws = self.map_ws if self.map_ws is not None else binding.alloc_block_map_workspace(self.d, DEV)
        binding.ss_block_map(self.d, slots, None, self.status, self.map_ws)
        self.ok()
        return indptr, R, slots

    def write(self, slots, tokens, positions):
        for l, c in enumerate(self.layers):
            k, v = self.values(l, 0, tokens, positions), self.values(l, 1, tokens, positions)
            binding.ss_kv_write(dict(c, total_rows=len(tokens), k_new=k, v_new=v, new_dtype=self.kv), slots)

    def prompts(self, rows, lengths):
        new = np.zeros(self.batch, int)
        new[rows] = lengths
        indptr, R, slots = self.step_arrays(new)
        tokens = self.rng.integers(0, VOCAB, R)
        positions = np.concatenate([np.arange(n) for n in new])
        self.write(slots, tokens, positions)
        for b in rows:
            self.tokens[b] = tokens[indptr[b]:indptr[b + 1]].tolist()
            self.next[b] = int(self.rng.integers(0, VOCAB))

    def fork(self, parent, child, length=None):
        n = len(parent)
        src, dst = i32(np.zeros(n)), i32(np.zeros(n))
        binding.ss_block_fork(self.d, i32(parent), i32(child), None if length is None else i32(length), src, dst, self.status, self.ws)
        binding.ss_block_copy(self.handle, src, dst)
        self.ok()
        for i, (p, c) in enumerate(zip(parent, child)):
            self.tokens[c] = self.tokens[p][:None if length is None else length[i]]
            self.next[c] = int(self.rng.integers(0, VOCAB))

    def drop(self, rows):
        keep = np.ones(self.batch, np.int32)
        keep[rows] = 0
        self.d["kv_len"] *= i32(keep)
        for b in rows:
            self.tokens[b], self.next[b] = [], None
        self.release()

    def release(self):
        binding.ss_block_release(self.d, self.status, self.ws)
        self.ok()

    def compact(self):
        N = self.d["num_blocks"]
        src, dst, moves = i32(np.zeros(N // 2)), i32(np.zeros(N // 2)), i32([0])
        binding.ss_block_compact(self.d, None, src, dst, moves, self.status, self.ws)
        binding.ss_block_copy(self.handle, src, dst, moves)
        self.ok()
        used = N - int(self.d["free_count"])
        for c in self.layers:      # what lies behind the blocks in use is nobody's
            c["k_cache"][used:] = float("nan")
            c["v_cache"][used:] = float("nan")

    def tree_step(self, widths):
        live = [b for b in range(self.batch) if self.next[b] is not None]
        new = np.zeros(self.batch, int)
        new[live] = widths[:len(live)]
        before = self.d["kv_len"].cpu().numpy().copy()
        indptr, R, slots = self.step_arrays(new)
        parent, tokens, positions, sees = np.full(R, -1, np.int32), np.zeros(R, np.int32), np.zeros(R, int), []
        logits = torch.from_numpy(self.rng.standard_normal((R, VOCAB)).astype(np.float32) * 2).to(torch.bfloat16)
        u = self.rng.random(R).astype(np.float32)
        u[u >= 1] = 0.0
        temp = np.where(np.arange(self.batch) % 3 == 0, 0.0, 0.9).astype(np.float32)
        for b in range(self.batch):
            r0, n = indptr[b], int(new[b])
            tree = ref.random_tree(n, self.rng, 12)
            sees.append(ref.ancestors(tree))
            for i, p in enumerate(tree):
                parent[r0 + i] = p
                tokens[r0 + i] = self.next[b] if i == 0 else self.rng.integers(0, VOCAB)
                positions[r0 + i] = before[b] + sees[b][i].sum() - 1
            for i in range(n):
                below = [c for c in range(i + 1, n) if tree[c] == i]
                if below and self.rng.random() < 0.8:
                    tokens[r0 + self.rng.choice(below)] = ref.draw(logits[r0 + i].double().numpy(), temp[b], u[r0 + i])[0]
        self.write(slots, tokens, positions)
        words = max(1, -(-int(new.max()) // 32))
        mask = np.zeros((R, words), np.uint32)
        for b in range(self.batch):
            if new[b]:
                mask[indptr[b]:indptr[b + 1]] = ref.pack(sees[b], words)
        q = torch.from_numpy(self.rng.standard_normal((R, HQ, D)).astype(np.float32)).to(DEV, torch.bfloat16 if self.kv == "bf16" else torch.float32)
        d = dict(self.layers[0], **self.d)
        d.update(num_q_heads=HQ, q_dtype=self.kv, q=q, node_mask=torch.from_numpy(mask.view(np.int32)).to(DEV), sees=sees, sm_scale=D ** -0.5)
        out, lse, ws = binding.alloc_tree_outputs(d, DEV, max_q_len=int(new.max()))
        for c in self.layers:
            binding.ss_tree_attn(dict(d, k_cache=c["k_cache"], v_cache=c["v_cache"]), out, lse, ws, max_q_len=int(new.max()))
        ref.check_tree(dict(d, k_cache=self.layers[-1]["k_cache"], v_cache=self.layers[-1]["v_cache"]), out, lse)
        v = dict(batch=self.batch, vocab=VOCAB, row_stride=VOCAB, logit_dtype="bf16", total_rows=R, q_indptr=self.d["q_indptr"], tree_parent=i32(parent), node_tokens=i32(tokens),
                 target_logits=logits.to(DEV), uniforms=torch.from_numpy(u).to(DEV), temperature=torch.from_numpy(temp).to(DEV))
        n_acc, emitted, nodes, logp, vws = binding.alloc_tree_verify_outputs(v, DEV)
        binding.ss_tree_verify(v, n_acc, emitted, nodes, logp, vws)
        want = ref.verify(logits.double().numpy(), indptr, R, parent, tokens, u, temp, 20)
        assert np.array_equal(n_acc.cpu().numpy(), want[0]) and np.array_equal(emitted.cpu().numpy(), want[1]) and np.array_equal(nodes.cpu().numpy(), want[2])
        for c in self.layers:
            binding.ss_kv_compact(dict(d, k_cache=c["k_cache"], v_cache=c["v_cache"]), nodes, n_acc)
        binding.ss_kv_commit(self.d["q_indptr"], n_acc, self.d["kv_len"])
        for b in live:
            n = int(want[0][b])
            self.tokens[b] += [self.next[b]] + want[1][b, :n].tolist()
            self.next[b] = int(want[1][b, n])
        self.release()
        return int(want[0].sum())

    def check(self):
        k = {name: self.d[name].cpu().numpy() for name in ("held", "kv_len", "shares")}
        ref.check_books(dict(k, table=self.d["block_table"].cpu().numpy(), free=self.d["free_ids"].cpu().numpy(), count=int(self.d["free_count"]), num_blocks=self.d["num_blocks"]))
        for b in range(self.batch):
            n = len(self.tokens[b])
            assert k["kv_len"][b] == n and k["held"][b] == blocks(n)
            if n == 0:
                continue
            ids = self.d["block_table"][b, :blocks(n)].long()
            for l, c in enumerate(self.layers):
                for side, name in enumerate(("k_cache", "v_cache")):
                    got = c[name][ids].transpose(1, 2).reshape(-1, HKV, D)[:n]
                    assert torch.equal(got, self.values(l, side, self.tokens[b], np.arange(n)).to(got.dtype)), (b, l, name)


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("seed", [0, 1])
def test_a_lane_of_shared_prompts_and_wide_trees(kv, seed):
    lane = Lane(14, 40, 330, kv, seed)
    lane.prompts([0, 3, 7], [200, 33, 160])
    lane.check()
    lane.fork([0, 0, 3, 7, 7], [1, 2, 5, 9, 12])
    lane.check()
    accepted = 0
    for step in range(3):
        accepted += lane.tree_step([40, 64, 1, 33, 22, 70, 5, 31])
        lane.check()
    lane.drop([0, 9])
    lane.check()
    lane.compact()
    lane.check()
    n = len(lane.tokens[1])
    lane.fork([1, 1, 12, 2], [0, 4, 9, 13], [n, n - 21, 160, 16])     # at an end, in the middle, at a block's end, behind one block
    lane.check()
    for step in range(3):
        accepted += lane.tree_step([90, 3, 32, 25, 48, 64, 2, 40, 11, 60])
        lane.check()
    lane.compact()
    lane.check()
    accepted += lane.tree_step([21] * 10)
    lane.check()
    lane.drop(list(range(14)))
    lane.check()
    assert accepted > 20 and int(lane.d["free_count"]) == 330
