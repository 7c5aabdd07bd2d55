"""A decode lane driven end to end through the library, on synthetic model outputs.

    python -m paper_2604_09562_amd.example [--steps N] [--batch B] [--layers L] [--tree] [--chunk C] [--wide N [--samples S]]

First the prompts are put into the empty cache, C new tokens of every request at a time:

  blocks      blocks for the new tokens, and where each goes                  ss_block_map
  write       their keys and values, once per layer                           ss_kv_write
  attention   over what is in the cache, once per layer                       ss_chunk_attn

Then each step does what a decode worker does around its model (whose projections and logits are stood in
for by seeded random tensors, there being no weights here):

  router      pick the worker for a new request from reported metrics         ss_route_select
  controller  per request, the next draft depth from its last acceptance     ss_depth_update
  blocks      blocks for the k+1 new tokens, those of rejected ones back      ss_block_map
  append      write the k+1 new tokens' keys/values into the paged cache      ss_kv_append
  attention   verify attention, once per layer; layers after the first        ss_spec_verify_attn
              reuse the first one's plan                                      (SS_BATCH_REUSE_PLAN)
  accept      acceptance walk and the draw of the next token                  ss_spec_accept, or for draft trees
                                                                              ss_spec_accept_tree_greedy / _sample + ss_kv_compact
  commit      new valid lengths                                               ss_kv_commit

and prints the accepted tokens per step.  With --wide every request is continued S times, in trees of up to N new tokens:

  forks       S requests that share the blocks of one prompt                  ss_block_fork, ss_block_copy
  blocks, write                                                               ss_block_map, ss_kv_write
  attention   of the trees' nodes, once per layer                             ss_tree_attn
  accept      the target's own draws, walked while a child carries them       ss_tree_verify
  commit      paths to their places, lengths, blocks of the rest back         ss_kv_compact, ss_kv_commit, ss_block_release

and half-way the last continuation of every request is dropped and the cache made whole again (ss_block_release, ss_block_compact, ss_block_copy).  Every device step runs in the library's kernels; this file
only moves arguments.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import binding, synth


def open_books(cache: dict, dev: str):
    """The cache's blocks, all free, and what the requests hold of them; returns the call that takes blocks for a step's new tokens."""
    i32 = lambda x: binding.to_device(np.asarray(x, dtype=np.int32), dev)  # noqa: E731
    cache.update(free_ids=i32(np.arange(cache["num_blocks"])), free_count=i32([cache["num_blocks"]]), held=i32(np.zeros(cache["batch"])),
                 block_table=torch.zeros_like(cache["block_table"]))
    status, ws = i32([0]), binding.alloc_block_map_workspace(cache, dev)

    def blocks(d, rows):
        slots = torch.empty(rows, dtype=torch.int32, device=dev)
        binding.ss_block_map(d, slots, None, status, ws)
        if int(status):      # (known before anything follows the table)
            raise RuntimeError(f"ss_block_map: status {int(status)}")
        return slots
    return blocks


def fill_prompts(cache: dict, lengths: np.ndarray, layers: int, chunk: int, blocks, rng, dev: str, verbose: bool) -> None:
    """Put prompts of these lengths into the empty cache, `chunk` tokens of every request at a time."""
    i32 = lambda x: binding.to_device(np.asarray(x, dtype=np.int32), dev)  # noqa: E731
    Hq, Hkv, D = cache["num_q_heads"], cache["num_kv_heads"], cache["head_dim"]
    done, chunks, t_prompt = np.zeros_like(lengths), 0, 0.0
    while (done < lengths).any():
        new = np.minimum(lengths - done, chunk)
        done += new
        q_indptr = np.concatenate([[0], np.cumsum(new)])
        R = int(q_indptr[-1])
        d = dict(cache, total_rows=R, q_dtype="bf16", new_dtype="bf16", kv_len=i32(done), q_indptr=i32(q_indptr))
        # queries, keys and values of a layer are parts of one product's rows
        wide = torch.from_numpy(rng.standard_normal((R, (Hq + 2 * Hkv) * D), dtype=np.float32)).to(dev, torch.bfloat16)
        d["q"], d["k_new"], d["v_new"] = (x.unflatten(1, (-1, D)) for x in wide.split([Hq * D, Hkv * D, Hkv * D], 1))
        out, lse, ws_c = binding.alloc_chunk_outputs(d, dev)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        slots = blocks(d, R)
        for _ in range(layers):
            binding.ss_kv_write(d, slots)
            binding.ss_chunk_attn(d, out, lse, ws_c)
        torch.cuda.synchronize()
        t_prompt += time.perf_counter() - t0
        chunks += 1
    if verbose:
        print(f"{int(lengths.sum())} prompt tokens in {chunks} chunks, {1e3 * t_prompt / max(chunks, 1):.3f} ms of device work per chunk ({layers} layers)")


def run(steps: int = 6, batch: int = 8, layers: int = 4, tree: bool = False, vocab: int = 32000, seed: int = 0,
        verbose: bool = True, sample: bool = False, chunk: int = 512) -> dict:
    dev = "cuda:0"
    torch.cuda.set_device(0)
    cfg = synth.CONFIGS[1].scaled(batch=batch, vocab=vocab, ctx=("uniform", 200, 1500))
    rng = np.random.default_rng(seed)

    # the router places a new request on one of four workers (host arithmetic)
    # (cache hit rate, memory utilisation, queue depth, active load, stale) as each worker reports them
    workers = [(float(rng.uniform(0, 1)), float(rng.uniform(0.2, 0.9)), int(rng.integers(0, 40)), float(rng.uniform(0, 1)), 0)
               for _ in range(4)]
    chosen = binding.ss_route_select(workers, q_max=64.0)

    # a paged cache with room for every step's tokens; `cur` = valid lengths before the step
    room = steps * (binding.SS_MAX_DEPTH + 1)
    host = synth.make_attention_inputs(cfg, seed=seed)
    cur = np.maximum(host["kv_len"].astype(np.int32) - room, 1)
    cache = binding.attention_to_device(host, dev)
    Hq, Hkv, D = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    ctrl = [binding.ss_depth_init() for _ in range(batch)]
    depth = np.full(batch, 4, dtype=np.int32)
    emitted, t_dev = 0, 0.0
    start_len = cur.copy()

    blocks = open_books(cache, dev)
    fill_prompts(cache, cur, layers, chunk, blocks, np.random.default_rng(seed + 1), dev, verbose)

    for step in range(steps):
        # ---- what the models would hand over: draft tokens/logits, queries and new keys/values per layer
        if tree and sample:
            acc = synth.make_tree_sample_inputs(cfg, seed=seed + step, depth=depth)
        elif tree:
            acc = synth.make_tree_accept_inputs(cfg, seed=seed + step, depth=depth, hit=0.7)
        else:
            acc = synth.make_accept_inputs(cfg, seed=seed + step, depth=depth)
        q_indptr, R = acc["q_indptr"], acc["total_rows"]
        mq = int(depth.max()) + 1
        d = dict(cache, depth=depth, total_rows=R, new_dtype="bf16")
        d["kv_len"] = binding.to_device((cur + depth + 1).astype(np.int32), dev)
        d["q_indptr"] = binding.to_device(q_indptr, dev)
        if tree:
            d["tree_mask"] = binding.to_device(acc["tree_mask"], dev)
        for name, heads in (("q", Hq), ("k_new", Hkv), ("v_new", Hkv)):
            d[name] = binding.to_device(synth.store(rng.standard_normal((R, heads, D), dtype=np.float32), "bf16"), dev)
        da = binding.accept_to_device(acc, dev)
        out, lse, ws = binding.alloc_attention_outputs(d, dev, max_q_len=mq)
        n_acc, toks, _, ws_a = binding.alloc_accept_outputs(da, dev)
        nodes = torch.empty((batch, binding.SS_MAX_DEPTH), dtype=torch.int32, device=dev)
        ws_t = binding.tree_sample_workspace(da, dev) if tree and sample else None

        # ---- the device side of the step
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        blocks(dict(d, tree_mask=None), R)
        binding.ss_kv_append(d, max_q_len=mq)
        for layer in range(layers):   # one cache stands in for every layer's; the batch metadata is shared
            binding.ss_spec_verify_attn(d, out, lse, ws, max_q_len=mq, reuse_plan=layer > 0)
        if tree:
            if sample:
                binding.ss_spec_accept_tree_sample(da, n_acc, toks, nodes, None, ws_t, max_q_len=mq)
            else:
                binding.ss_spec_accept_tree_greedy(da, n_acc, toks, nodes, ws_a, max_q_len=mq)
            binding.ss_kv_compact(d, nodes, n_acc, max_q_len=mq)
        else:
            binding.ss_spec_accept(da, n_acc, toks, None, ws_a, max_q_len=mq)
        binding.ss_kv_commit(d["q_indptr"], n_acc, d["kv_len"])
        torch.cuda.synchronize()
        t_dev += time.perf_counter() - t0

        # ---- feedback: the controller turns each request's acceptance into its next depth
        n = n_acc.cpu().numpy()
        cur = d["kv_len"].cpu().numpy()
        load, tput = 0.3, 300.0
        for b in range(batch):
            a = n[b] / depth[b] if depth[b] else 0.0
            depth[b] = binding.ss_depth_update(ctrl[b], float(a), load, tput)[3]
        emitted += int(n.sum()) + batch
        if verbose:
            print(f"step {step}: accepted {n.tolist()} -> next depths {depth.tolist()}")
    if verbose:
        print(f"router chose worker {chosen}; {emitted} tokens emitted in {steps} steps, "
              f"{1e3 * t_dev / steps:.3f} ms of device work per step ({layers} layers)")
    return dict(chosen=chosen, emitted=emitted, depths=depth.copy(), kv_len=cur, start_len=start_len)


def wide_trees(rng, live, nodes, drawn, vocab):
    """Trees of up to `nodes` new tokens for the requests in `live`, `drawn` at their roots: (new tokens of each, q_indptr, parents, tokens, masks)."""
    new = np.where(live, rng.integers(min(2, nodes), nodes + 1, len(live)), 0)
    q_indptr = np.concatenate([[0], np.cumsum(new)])
    R, words = int(q_indptr[-1]), -(-nodes // 32)
    parent, tokens, mask = np.full(R, -1, np.int32), rng.integers(0, vocab, R).astype(np.int32), np.zeros((R, words), np.uint32)
    for b, r0 in enumerate(q_indptr[:-1]):
        for i in range(new[b]):
            if i == 0:
                tokens[r0] = drawn[b]
            else:
                parent[r0 + i] = rng.integers(max(i - 8, 0), i)
                mask[r0 + i] = mask[r0 + parent[r0 + i]]      # a node attends its ancestors
            mask[r0 + i, i // 32] |= np.uint32(1 << i % 32)   # and itself
    return new, q_indptr, parent, tokens, mask


def run_wide(steps: int = 6, batch: int = 4, layers: int = 4, nodes: int = 48, samples: int = 3, vocab: int = 32000, seed: int = 0, chunk: int = 512,
             temperature: float = 0.8, verbose: bool = True) -> dict:
    """`samples` continuations of each of `batch` prompts, in draft trees of up to `nodes` new tokens."""
    dev = "cuda:0"
    torch.cuda.set_device(0)
    i32 = lambda x: binding.to_device(np.asarray(x, dtype=np.int32), dev)  # noqa: E731
    rows = batch * samples
    cfg = synth.CONFIGS[1].scaled(batch=rows, vocab=vocab, ctx=("uniform", 200, 1500))
    rng = np.random.default_rng(seed)
    host = synth.make_attention_inputs(cfg, seed=seed)
    room = nodes + steps * (binding.SS_MAX_DEPTH + 1)
    prompts = np.where(np.arange(rows) % samples == 0, np.maximum(host["kv_len"].astype(np.int32) - room, 1), 0).astype(np.int32)
    cache = binding.attention_to_device(host, dev)
    columns = -(-(int(prompts.max()) + room) // 16)
    cache.update(max_blocks_per_seq=columns, block_table=torch.zeros((rows, columns), dtype=torch.int32, device=dev))
    Hq, Hkv, D, N = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim, cache["num_blocks"]
    blocks = open_books(cache, dev)
    fill_prompts(cache, prompts, layers, chunk, blocks, np.random.default_rng(seed + 1), dev, verbose)
    cache.update(kv_len=i32(prompts), shares=i32(np.zeros(N)))
    handle = binding.cache_layers([cache])      # (one cache stands in for every layer's)
    status, ws = i32([0]), binding.alloc_block_share_workspace(cache, dev, num_forks=rows)

    def ok(call):
        if int(status):
            raise RuntimeError(f"{call}: status {int(status)}")

    # ---- the continuations share their prompt's blocks; a block that is not full is copied
    children = np.flatnonzero(prompts == 0)
    if len(children):
        src, dst = i32(np.zeros(len(children))), i32(np.zeros(len(children)))
        binding.ss_block_fork(cache, i32(children // samples * samples), i32(children), None, src, dst, status, ws)
        binding.ss_block_copy(handle, src, dst)
        ok("ss_block_fork")
    start_len = cache["kv_len"].cpu().numpy()
    live, drawn = np.ones(rows, bool), rng.integers(0, vocab, rows)
    emitted, moved, t_dev = np.zeros(rows, int), 0, 0.0
    for step in range(steps):
        if step == steps // 2 and samples > 1:
            live[samples - 1::samples] = False
            cache["kv_len"] *= i32(live)
            binding.ss_block_release(cache, status, ws)
            ok("ss_block_release")
            src, dst, moves = i32(np.zeros(N // 2)), i32(np.zeros(N // 2)), i32([0])
            binding.ss_block_compact(cache, None, src, dst, moves, status, ws)
            binding.ss_block_copy(handle, src, dst, moves)
            ok("ss_block_compact")
            moved = int(moves)
        # ---- what the models would hand over
        new, q_indptr, parent, tokens, mask = wide_trees(rng, live, nodes, drawn, vocab)
        R = int(q_indptr[-1])
        d = dict(cache, total_rows=R, q_dtype="bf16", new_dtype="bf16", kv_len=cache["kv_len"] + i32(new), q_indptr=i32(q_indptr),
                 node_mask=binding.to_device(mask.view(np.int32), dev))
        wide = torch.from_numpy(rng.standard_normal((R, (Hq + 2 * Hkv) * D), dtype=np.float32)).to(dev, torch.bfloat16)
        d["q"], d["k_new"], d["v_new"] = (x.unflatten(1, (-1, D)) for x in wide.split([Hq * D, Hkv * D, Hkv * D], 1))
        logits = torch.from_numpy(rng.standard_normal((R, vocab), dtype=np.float32)).to(dev, torch.bfloat16)
        has_child = np.flatnonzero(parent >= 0)      # the target thinks well of some of the drafts
        below = has_child[rng.random(len(has_child)) < 0.3]
        root = np.repeat(q_indptr[:-1], new)
        logits[torch.from_numpy(root[below] + parent[below]).to(dev), torch.from_numpy(tokens[below].astype(np.int64)).to(dev)] = 12.0
        v = dict(batch=rows, vocab=vocab, row_stride=vocab, logit_dtype="bf16", total_rows=R, q_indptr=d["q_indptr"], tree_parent=i32(parent), node_tokens=i32(tokens),
                 target_logits=logits, uniforms=torch.from_numpy(rng.random(R, dtype=np.float32)).to(dev), temperature=None, temperature_scalar=temperature)
        out, lse, ws_t = binding.alloc_tree_outputs(d, dev, max_q_len=nodes)
        n_acc, toks, accepted, logp, ws_v = binding.alloc_tree_verify_outputs(v, dev)

        # ---- the device side of the step
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        slots = blocks(d, R)
        for _ in range(layers):
            binding.ss_kv_write(d, slots)
            binding.ss_tree_attn(d, out, lse, ws_t, max_q_len=nodes)
        binding.ss_tree_verify(v, n_acc, toks, accepted, logp, ws_v)
        binding.ss_kv_compact(d, accepted, n_acc, max_q_len=nodes)      # (once: one cache stands in for every layer's)
        binding.ss_kv_commit(d["q_indptr"], n_acc, d["kv_len"])
        binding.ss_block_release(d, status, ws)
        torch.cuda.synchronize()
        t_dev += time.perf_counter() - t0
        ok("ss_block_release")

        cache["kv_len"] = d["kv_len"]
        n = np.where(live, n_acc.cpu().numpy(), 0)
        drawn = toks.cpu().numpy()[np.arange(rows), n]
        emitted += np.where(live, n + 1, 0)
        if verbose:
            print(f"step {step}: {R} nodes, accepted {n[live].tolist()}, mean log-probability {float(logp[torch.from_numpy(live).to(dev), 0].mean()):.2f}")
    held = int(cache["held"].sum())
    if verbose:
        print(f"{int(emitted.sum())} tokens emitted in {steps} steps, {1e3 * t_dev / max(steps, 1):.3f} ms of device work per step ({layers} layers); "
              f"{held} blocks held, {N - int(cache['free_count'])} in use, {moved} moved")
    return dict(emitted=emitted, live=live, kv_len=cache["kv_len"].cpu().numpy(), start_len=start_len, held=held, used=N - int(cache["free_count"]))


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--tree", action="store_true", help="tree-shaped drafts (greedy acceptance unless --sample)")
    ap.add_argument("--chunk", type=int, default=512, help="new tokens of a request's prompt at a time")
    ap.add_argument("--sample", action="store_true", help="with --tree: the sampled acceptance walk")
    ap.add_argument("--wide", type=int, default=0, metavar="N", help="draft trees of up to N new tokens, verified by the target's own draws")
    ap.add_argument("--samples", type=int, default=3, help="with --wide: continuations of each prompt, which share its blocks")
    a = ap.parse_args()
    if a.wide:
        run_wide(a.steps, a.batch, a.layers, a.wide, a.samples, chunk=a.chunk)
        return
    run(a.steps, a.batch, a.layers, a.tree, sample=a.sample, chunk=a.chunk)


if __name__ == "__main__":
    main()
