"""ss_kv_compact behind trees of any width: the accepted nodes' keys and values move to where a chain would stand, to the bit; nothing follows ids or lengths that cannot be."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from .prefill_ref import BLOCK, DEV, TORCH

pytestmark = pytest.mark.gpu

HKV, D = 3, 64


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def batch(kv, lengths, seed, spare=3):
    """A cache of any bits (finite ones), requests of (new tokens, length), paths of up to 20 of their nodes."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    held = [-(-n // BLOCK) for _, n in lengths]
    N, width = sum(held) + spare, max(held) + 2
    ids, table, at = rng.permutation(N), np.full((len(lengths), width), -1, np.int64), 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    x = [torch.randn((N, HKV, BLOCK, D), device=DEV, generator=gen).to(TORCH[kv]) for _ in range(2)]
    s = [torch.rand((N, HKV), device=DEV, generator=gen) * 4 + 0.01 if kv == "fp8" else None for _ in range(2)]
    nodes, n_acc = np.full((len(lengths), 20), -1, np.int64), np.zeros(len(lengths), np.int64)
    for b, (q, _) in enumerate(lengths):
        n_acc[b] = rng.integers(0, min(q, 21)) if q > 0 else 0
        nodes[b, :n_acc[b]] = np.sort(rng.permutation(np.arange(1, max(q, 1)))[:n_acc[b]])
    d = dict(num_blocks=N, block_size=BLOCK, num_kv_heads=HKV, head_dim=D, kv_dtype=kv, k_cache=x[0], v_cache=x[1], k_scale=s[0], v_scale=s[1], batch=len(lengths),
             max_blocks_per_seq=width, block_table=i32(table), kv_len=i32([n for _, n in lengths]), q_indptr=i32(np.concatenate([[0], np.cumsum([q for q, _ in lengths])])),
             total_rows=int(sum(q for q, _ in lengths)))
    return d, nodes, n_acc


def moved(d, nodes, n_acc, lengths, only=None):
    """The caches behind the moves, one after the other in path order."""
    table, out = d["block_table"].cpu().numpy(), []
    for x, s in ((d["k_cache"], d["k_scale"]), (d["v_cache"], d["v_scale"])):
        y = x.clone()
        for b, (q, n) in enumerate(lengths):
            if only is not None and b not in only:
                continue
            for j, node in enumerate(nodes[b, :n_acc[b]], 1):
                src, dst = n - q + int(node), n - q + j
                bs, bd = int(table[b, src // BLOCK]), int(table[b, dst // BLOCK])
                row = y[bs, :, src % BLOCK].clone()
                if s is not None and bs != bd:
                    z = row.float() * s[bs][:, None] / s[bd][:, None]
                    row = z.clamp(-448, 448).to(row.dtype)
                y[bd, :, dst % BLOCK] = row
        out.append(y)
    return out


def check(d, want):
    for x, w in zip((d["k_cache"], d["v_cache"]), want):
        assert torch.equal(x.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("lengths", [[(1, 1), (2, 2), (64, 64), (65, 300), (33, 33)], [(130, 500), (22, 40), (0, 77), (48, 4096)]])
def test_paths_of_wide_trees(kv, lengths):
    for seed in range(3):
        d, nodes, n_acc = batch(kv, lengths, seed)
        want = moved(d, nodes, n_acc, lengths)
        binding.ss_kv_compact(d, i32(nodes), i32(n_acc), max_q_len=130 if seed else 0)
        torch.cuda.synchronize()
        check(d, want)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_ids_and_lengths_that_cannot_be_are_not_followed(kv):
    lengths = [(40, 100), (64, 90), (50, 200), (30, 64)]
    for change in ("ids", "long", "longest", "short"):
        d, nodes, n_acc = batch(kv, lengths, 5)
        n_acc[1:3] = 18
        for b in (1, 2):
            nodes[b, :18] = np.arange(2, 20)     # every node moves
        want = moved(d, nodes, n_acc, lengths, only=(0, 3))
        if change == "ids":
            d["block_table"][1] = torch.tensor([-1, d["num_blocks"], 2 ** 31 - 1, -2 ** 31] * 9, dtype=torch.int32, device=DEV)[:d["max_blocks_per_seq"]]
            d["block_table"][2] = -7
        else:
            d["kv_len"][1] = {"long": d["max_blocks_per_seq"] * BLOCK + 1, "longest": 2 ** 31 - 1, "short": 63}[change]
            d["kv_len"][2] = {"long": 2 ** 30, "longest": 2 ** 31 - 1, "short": -2 ** 31}[change]
        binding.ss_kv_compact(d, i32(nodes), i32(n_acc))
        torch.cuda.synchronize()
        check(d, want)
