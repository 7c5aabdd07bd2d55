"""Wide draft trees over caches that requests share, as cases that can be timed and checked: attention of a tree of drafted tokens,
verification of the tree against the target's distributions from given uniforms, and forking, releasing and compacting the blocks of a
cache.

A case is a dict of plain values; `listed()` gives the fixed ones, `draw(rng)` more of the same ranges.  `prepare(case, seed)` puts on the
GPU what a serving program holds before the call, `run(state)` makes one pass through an operator: the public calls of
`paper_2604_09562_amd.binding` where `own` is true, plain torch operations where it is not (attention in 32 bits, draws in 64).
`exact(case, seed)` gives attention's results and the tokens' log-probabilities in 64 bits; everything else is whole numbers or copies.

Lengths and trees follow from the case alone (its "sizes" number); the seed shuffles the requests and makes every value.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 16          # tokens per cache block
FP8_MAX = 448.0     # largest finite e4m3 value
MAX_DEPTH = 20      # accepted tokens a request's row of nodes has room for

_ESZ = {"f32": 4, "bf16": 2, "fp8": 1}
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def _attn(name, batch, n_lo, n_hi, ctx_lo, ctx_hi, hq, hkv, d, kv, q="bf16", sizes=1):
    c = dict(kind="attn", batch=batch, n_lo=n_lo, n_hi=n_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, hq=hq, hkv=hkv, head_dim=d, kv=kv, q=q,
             sizes=sizes)
    return dict(name=name, **c) if name else c


def _verify(name, batch, n_lo, n_hi, depth, vocab, logits, temperature, sizes=1):
    c = dict(kind="verify", batch=batch, n_lo=n_lo, n_hi=n_hi, depth=depth, vocab=vocab, logits=logits, temperature=temperature, sizes=sizes)
    return dict(name=name, **c) if name else c


def _blocks_case(kind, name, parents, children, len_lo, len_hi, layers, hkv, d, kv, spare=0.1, sizes=1):
    c = dict(kind=kind, parents=parents, children=children, len_lo=len_lo, len_hi=len_hi, layers=layers, hkv=hkv, head_dim=d, kv=kv,
             spare=spare, sizes=sizes)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one request with a small tree behind a short prompt: launches and latency decide
        _attn("tree_25_b1", 1, 25, 25, 300, 300, 32, 8, 128, "bf16"),
        # an ordinary micro-batch with trees of up to 64 nodes
        _attn("tree_64_b16", 16, 33, 64, 512, 8192, 32, 8, 128, "bf16"),
        # a large model with an 8-bit cache, eight query heads per KV head and long contexts
        _attn("tree_70b_fp8_b8", 8, 30, 60, 4096, 16384, 64, 8, 128, "fp8"),
        # the small float32 configuration with 64-wide heads
        _attn("tree_f32_b4", 4, 10, 40, 64, 512, 8, 2, 64, "f32", q="f32"),
        # one request's tree against a small vocabulary
        _verify("verify_b1", 1, 25, 25, 6, 32000, "f32", 1.0),
        # a full micro-batch of wide trees against a large one
        _verify("verify_wide_b64", 64, 24, 64, 8, 128256, "bf16", 0.8),
        # four samples of one prompt: three forks, every layer's last block copied
        _blocks_case("fork", "fork_samples_b1", 1, 3, 500, 500, 16, 8, 128, "bf16"),
        # a step of a search that keeps several continuations of many requests, 8-bit cache
        _blocks_case("fork", "fork_beams_b32", 32, 3, 256, 4096, 8, 8, 128, "fp8"),
        # an ordinary step: some forks of sixteen requests are dropped, others give drafts' blocks back
        _blocks_case("release", "release_step_b64", 16, 3, 256, 4096, 0, 8, 128, "bf16"),
        # the end of many long requests that shared their prompts
        _blocks_case("release", "release_many_b256", 64, 3, 1024, 16384, 0, 8, 128, "bf16"),
        # a small cache after a few requests have gone
        _blocks_case("compact", "compact_small", 6, 0, 64, 700, 4, 8, 128, "bf16", spare=0.5),
        # a cache of which half is free, in pieces, made whole again
        _blocks_case("compact", "compact_half_free", 24, 1, 256, 4096, 8, 8, 128, "bf16", spare=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: any batch, tree, grouping, cache type and length; bounded in cost."""
    while True:
        kind = rng.choice(["attn"] * 5 + ["small", "verify", "verify", "fork", "release", "compact"])
        sizes = rng.randrange(1, 1 << 20)
        n_hi = _log_int(rng, 1, 256)
        n_lo = _log_int(rng, max(1, n_hi // 4), n_hi)
        hkv = rng.choice([1, 2, 4, 8, 8])
        if kind == "attn":
            ctx_hi = rng.choice([0, _log_int(rng, 16, 32768), _log_int(rng, 16, 32768), _log_int(rng, 16, 32768)])
            c = _attn(None, _log_int(rng, 1, 32), n_lo, n_hi, rng.randint(0, ctx_hi), ctx_hi, hkv * rng.choice([1, 2, 4, 4, 5, 7, 8, 8]), hkv,
                      rng.choice([128, 128, 128, 64]), rng.choice(["bf16", "bf16", "fp8"]), sizes=sizes)
            if c["batch"] * n_hi * (n_hi + ctx_hi) * c["hq"] > 5e8 or work(c)["flops"] > 8.0e10 or work(c)["bytes"] > 4.0e8:
                continue
        elif kind == "small":    # float32 on either side: small calls only
            ctx_hi = rng.choice([0, _log_int(rng, 16, 1000)])
            c = _attn(None, _log_int(rng, 1, 8), min(n_lo, 64), min(n_hi, 64), rng.randint(0, ctx_hi), ctx_hi, hkv * rng.choice([1, 2, 4, 7]), hkv,
                      rng.choice([64, 128]), rng.choice(["f32", "f32", "bf16"]), q="f32", sizes=sizes)
        elif kind == "verify":
            c = _verify(None, _log_int(rng, 1, 64), n_lo, n_hi, rng.randint(1, 12), _log_int(rng, 1000, 152064), rng.choice(["bf16", "bf16", "f32"]),
                        rng.choice([0.0, 0.7, 0.8, 1.0, 1.3]), sizes=sizes)
            if sum(n for n, _ in _trees(c)) * c["vocab"] * _ESZ[c["logits"]] > 7.0e8 or work(c)["bytes"] > 5.0e7:
                continue
        else:
            len_hi = _log_int(rng, 1, 8192)
            c = _blocks_case(kind, None, _log_int(rng, 1, 64), rng.randint(0 if kind != "fork" else 1, 4), _log_int(rng, max(1, len_hi // 16), len_hi), len_hi,
                             0 if kind == "release" else _log_int(rng, 1, 8), hkv, rng.choice([128, 128, 64]), rng.choice(["bf16", "bf16", "fp8", "f32"]),
                             rng.choice([0.1, 0.3, 1.0]), sizes=sizes)
            p = _block_plan(c)
            if p["total"] * c["layers"] * _block_bytes(c) > 2.5e9 or work(c)["bytes"] > (5.0e8 if kind == "compact" else 9.0e7):
                continue
        return c


# ---------------------------------------------------------------------------------------------------
# sizes: from the case alone
# ---------------------------------------------------------------------------------------------------
def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _sizes(case):
    """[(nodes, cache length with them)] per request, before shuffling."""
    rng = random.Random(case["sizes"])
    out = []
    for _ in range(case["batch"]):
        n = _log_int(rng, case["n_lo"], case["n_hi"])
        out.append((n, n + rng.randint(case["ctx_lo"], case["ctx_hi"])))
    return out


def _tree(rng, n, depth):
    """Parents of a random tree of n nodes, -1 for the root: any earlier node that is not too deep, recent ones more often."""
    parent, level = [-1], [0]
    for i in range(1, n):
        while True:
            p = max(rng.randrange(i), rng.randrange(i)) if rng.random() < 0.5 else rng.randrange(i)
            if level[p] < depth:
                break
        parent.append(p)
        level.append(level[p] + 1)
    return parent


def _trees(case):
    """[(nodes, (parents, path))] per request: a tree and how far into it the target's own tokens lead."""
    rng = random.Random(case["sizes"])
    out = []
    for _ in range(case["batch"]):
        n = _log_int(rng, case["n_lo"], case["n_hi"])
        parent = _tree(rng, n, case["depth"])
        path, cur = [], 0
        while rng.random() < 0.75:       # three of four draws are among the drafted children
            below = [c for c in range(cur + 1, n) if parent[c] == cur]
            if not below:
                break
            cur = rng.choice(below)
            path.append(cur)
        out.append((n, (parent, path)))
    return out


def _block_bytes(case):
    """Bytes of a block's keys and values in one layer."""
    return 2 * case["hkv"] * (BLOCK * case["head_dim"] * _ESZ[case["kv"]] + (4 if case["kv"] == "fp8" else 0))


def _block_plan(case):
    """A cache with requests that share blocks, before the call; logical ids, which the seed permutes.

    rows: (blocks in order, length) per request; shares: holders beyond the first per id; total: blocks of the cache, those from used
    on being free; forks: (parent, child, length).  For "release" the lengths are those after the requests have been shortened."""
    rng = random.Random(case["sizes"] + 7)
    kids, kind = case["children"], case["kind"]
    rows, shares, used, forks = [], [], 0, []
    for _ in range(case["parents"]):
        n = _log_int(rng, case["len_lo"], case["len_hi"])
        ids = list(range(used, used + _blocks(n)))
        used += len(ids)
        shares += [0] * len(ids)
        first = len(rows)
        rows.append((ids, n))
        for _ in range(kids):
            at = n if rng.random() < 0.75 else rng.randint(1, n)     # mostly at the end, some at an earlier token
            if kind == "fork":
                forks.append((first, len(rows), at))
                rows.append(([], 0))
                continue
            mine = ids[:at // BLOCK]        # forked some time ago, and grown since
            for x in mine:
                shares[x] += 1
            more = at + rng.randint(1, 64)
            fresh = _blocks(more) - len(mine)
            rows.append((mine + list(range(used, used + fresh)), more))
            used += fresh
            shares += [0] * fresh
    if kind == "release":
        out = []
        for ids, n in rows:
            u = rng.random()
            if u < 0.5:
                n = 0                                   # ended, or dropped from the search
            elif u < 0.75:
                n = max(n - rng.randint(1, 40), 1)       # rejected drafts
            out.append((ids, n))
        rows = out
    free = max(int(used * case["spare"]), len(forks)) + 2
    return dict(rows=rows, shares=shares, total=used + free, used=used, forks=forks)


def work(case):
    if case["kind"] == "attn":
        sizes = _sizes(case)
        hq, hkv, d, es = case["hq"], case["hkv"], case["head_dim"], _ESZ[case["kv"]]
        rows, blocks = sum(n for n, _ in sizes), sum(_blocks(m) for _, m in sizes)
        words = max((n + 31) // 32 for n, _ in sizes)
        b = sum(m for _, m in sizes) * hkv * d * 2 * es + blocks * 4 + rows * (hq * (2 * d * _ESZ[case["q"]] + 4) + 4 * words) + 8 * len(sizes)
        if case["kv"] == "fp8":
            b += blocks * hkv * 8
        # scores and outputs of the context; of the new tokens a node's ancestors only, counted as one
        return {"bytes": b, "flops": sum(4 * d * hq * n * (m - n + 1) for n, m in sizes)}
    if case["kind"] == "verify":
        trees = _trees(case)
        draws = sum(len(path) + 1 for _, (_, path) in trees)
        return {"bytes": draws * case["vocab"] * _ESZ[case["logits"]] + sum(n for n, _ in trees) * 8 + len(trees) * 4 * (2 * MAX_DEPTH + 3),
                "flops": draws * case["vocab"] * 3}
    p = _block_plan(case)
    if case["kind"] == "fork":
        entries = sum(_blocks(n) for _, _, n in p["forks"])
        copies = sum(1 for _, _, n in p["forks"] if n % BLOCK)
        return {"bytes": entries * 16 + copies * 2 * case["layers"] * _block_bytes(case) + len(p["forks"]) * 32, "flops": 0}
    if case["kind"] == "release":
        given = sum(max(len(ids) - _blocks(n), 0) for ids, n in p["rows"])
        return {"bytes": given * 16 + len(p["rows"]) * 12, "flops": 0}
    moved = p["used"] * (p["total"] - p["used"]) // p["total"]     # of a random order, in the mean
    return {"bytes": moved * 2 * case["layers"] * _block_bytes(case) + 8 * sum(len(ids) for ids, _ in p["rows"]) + 12 * p["total"], "flops": 0}


# ---------------------------------------------------------------------------------------------------
# inputs: from case and seed
# ---------------------------------------------------------------------------------------------------
class _State:
    pass


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _order(n, seed):
    order = list(range(n))
    random.Random(seed * 7919 + 1).shuffle(order)
    return order


def _cache_values(shape, dtype, gen):
    """N(0,1) keys or values in storage format: (data, per-block scale or None)."""
    if dtype != "fp8":
        return torch.randn(shape, dtype=_TORCH[dtype], device=DEV, generator=gen), None
    scale = torch.rand(shape[:2], device=DEV, generator=gen) * 0.09 + 0.01
    x = torch.randn(shape, device=DEV, generator=gen) / scale[:, :, None, None]
    return x.clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn), scale


def _at(cache, ids):
    """Blocks of a cache, of any type (8-bit ones are indexed as bytes)."""
    return cache.view(torch.uint8)[ids].view(cache.dtype) if cache.dtype == torch.float8_e4m3fn else cache[ids]


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _mask_words(parents, words):
    """Per node its own bit and its ancestors', as signed 32-bit words."""
    rows = []
    for i, p in enumerate(parents):
        bits = (rows[p] if p >= 0 else 0) | 1 << i
        rows.append(bits)
    return [[((r >> 32 * w & 0xffffffff) ^ 0x80000000) - 0x80000000 for w in range(words)] for r in rows]


def _inputs_attn(s, case, seed, gen):
    hq, hkv, d = case["hq"], case["hkv"], case["head_dim"]
    sizes = _sizes(case)
    rng = random.Random(case["sizes"] + 3)
    trees = [_tree(rng, n, 10) for n, _ in sizes]
    order = _order(len(sizes), seed)
    sizes, trees = [sizes[i] for i in order], [trees[i] for i in order]
    s.batch, s.max_q = len(sizes), max(n for n, _ in sizes)
    indptr = _starts([n for n, _ in sizes])
    s.rows, s.words = indptr[-1], (s.max_q + 31) // 32
    s.kv_len, s.q_indptr = _int32([m for _, m in sizes]), _int32(indptr)
    s.mask = _int32([w for t in trees for w in _mask_words(t, s.words)])
    counts = [_blocks(m) for _, m in sizes]
    used = sum(counts)
    s.num_blocks = used + used // 10 + 1
    perm = torch.randperm(s.num_blocks, generator=torch.Generator().manual_seed(seed))[:used].to(torch.int32)
    table = torch.full((s.batch, max(counts)), -1, dtype=torch.int32)
    for b, at in enumerate(_starts(counts)[:-1]):
        table[b, :counts[b]] = perm[at:at + counts[b]]
    shape = (s.num_blocks, hkv, BLOCK, d)
    s.k, s.k_scale = _cache_values(shape, case["kv"], gen)
    s.v, s.v_scale = _cache_values(shape, case["kv"], gen)
    for cache in (s.k, s.v):                # what stands behind a request's last token is of no one
        raw, big = (cache.view(torch.uint8), 0x7E) if case["kv"] == "fp8" else (cache, 1.0e4)
        for b, (_, m) in enumerate(sizes):
            if m % BLOCK:
                raw[int(table[b, _blocks(m) - 1]), :, m % BLOCK:] = big
    # the queries as a model has them: part of what its projection of queries, keys and values wrote; heads differ in how sharply they attend
    sharp = torch.rand((1, hq, 1), device=DEV, generator=gen) * 3.0 + 1.0
    qkv = torch.empty((s.rows, (hq + 2 * hkv) * d), dtype=_TORCH[case["q"]], device=DEV)
    qkv[:, :hq * d] = (torch.randn((s.rows, hq, d), device=DEV, generator=gen) * sharp).view(s.rows, hq * d)
    s.q = qkv[:, :hq * d].unflatten(1, (hq, d))
    s.table = table.to(DEV)
    s.scale = 1.0 / math.sqrt(d)


def _handles_attn(s, binding):
    case = s.case
    s.d = dict(batch=s.batch, num_q_heads=case["hq"], num_kv_heads=case["hkv"], head_dim=case["head_dim"], block_size=BLOCK, num_blocks=s.num_blocks,
               max_blocks_per_seq=s.table.shape[1], total_rows=s.rows, kv_dtype=case["kv"], q_dtype=case["q"], kv_len=s.kv_len,
               q_indptr=s.q_indptr, block_table=s.table, k_cache=s.k, v_cache=s.v, k_scale=s.k_scale, v_scale=s.v_scale, q=s.q,
               node_mask=s.mask, sm_scale=s.scale)
    s.out, s.lse, s.ws = binding.alloc_tree_outputs(s.d, DEV, max_q_len=s.max_q)


def _draw_tokens(rows, temperature, u):
    """The token that each row's uniform draws, and the logarithm of its probability: the first whose running sum of exp((x - max) / T)
    exceeds u times the whole; at temperature 0 the largest entry's, the first of several, with probability one."""
    x = rows.double()
    if temperature == 0.0:
        return x.argmax(-1), torch.zeros((x.shape[0],), device=DEV)
    x = (x - x.amax(-1, keepdim=True)) / temperature
    c = x.exp().cumsum_(-1)
    y = (c > u.double()[:, None] * c[:, -1:]).int().argmax(-1)
    return y, (x.gather(1, y[:, None])[:, 0] - c[:, -1].log()).float()


def _inputs_verify(s, case, seed, gen):
    trees = _trees(case)
    trees = [trees[i] for i in _order(len(trees), seed)]
    V = case["vocab"]
    s.batch, s.max_q = len(trees), max(n for n, _ in trees)
    indptr = _starts([n for n, _ in trees])
    s.rows = indptr[-1]
    s.row_stride = (V + 7) // 8 * 8
    s.q_indptr = _int32(indptr)
    s.logits = torch.empty((s.rows, s.row_stride), dtype=_TORCH[case["logits"]], device=DEV)
    for lo in range(0, s.rows, 256):
        x = torch.randn((min(256, s.rows - lo), s.row_stride), device=DEV, generator=gen) * 2.5
        x[:, ::97] += 5.0                       # a few candidates stand out
        s.logits[lo:lo + x.shape[0]] = x.to(s.logits.dtype)
    s.u = torch.rand((s.rows,), device=DEV, generator=gen)
    s.parent = _int32([p for _, (parent, _) in trees for p in parent])
    # Drafted tokens: candidates that are likely under the parent; on the planned path the one that the target draws there, elsewhere another.
    local = torch.cat([torch.full((n,), indptr[b]) for b, (n, _) in enumerate(trees)]).to(DEV)
    rank = torch.rand((s.rows,), device=DEV, generator=gen)
    s.tokens = ((rank * (V // 97)).long() * 97).clamp_(max=V - 1)
    above = (s.parent.clamp(min=0) + local).long()
    drawn = torch.empty((s.rows,), dtype=torch.int64, device=DEV)
    for lo in range(0, s.rows, 256):
        drawn[lo:lo + 256] = _draw_tokens(s.logits[lo:lo + 256, :V], case["temperature"], s.u[lo:lo + 256])[0]
    s.tokens = torch.where(s.tokens == drawn[above], (s.tokens + 1) % V, s.tokens)
    path = torch.tensor([indptr[b] + c for b, (_, (_, p)) in enumerate(trees) for c in p], dtype=torch.int64, device=DEV)
    s.tokens[path] = drawn[above[path]]
    s.tokens = s.tokens.to(torch.int32)
    s.depth = case["depth"]


def _handles_verify(s, binding):
    case = s.case
    s.d = dict(batch=s.batch, vocab=case["vocab"], row_stride=s.row_stride, logit_dtype=case["logits"], total_rows=s.rows, q_indptr=s.q_indptr,
               tree_parent=s.parent, node_tokens=s.tokens, target_logits=s.logits, uniforms=s.u, temperature=None,
               temperature_scalar=case["temperature"])
    s.n, s.out, s.nodes, s.logp, s.ws = binding.alloc_tree_verify_outputs(s.d, DEV)


def _inputs_blocks(s, case, seed, gen):
    p = _block_plan(case)
    order = _order(len(p["rows"]), seed)
    where = {old: new for new, old in enumerate(order)}
    perm = torch.randperm(p["total"], generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    rows = [p["rows"][i] for i in order]
    s.batch, s.num_blocks = len(rows), p["total"]
    width = max(max(len(ids) for ids, _ in rows), max([_blocks(n) for _, _, n in p["forks"]], default=0), 1)
    table = torch.full((s.batch, width), -1, dtype=torch.int32)
    for b, (ids, _) in enumerate(rows):
        table[b, :len(ids)] = perm[torch.tensor(ids, dtype=torch.int64)]
    shares = torch.zeros((p["total"],), dtype=torch.int32)
    shares[perm[:p["used"]].long()] = torch.tensor(p["shares"], dtype=torch.int32)
    count = p["total"] - p["used"]
    free = torch.full((p["total"],), -1, dtype=torch.int32)
    free[:count] = perm[p["used"]:]
    held, kv_len = [len(ids) for ids, _ in rows], [n for _, n in rows]
    # all of the cache's books, as they are before the call: each pass starts from them
    parts = [table.view(-1), torch.tensor(held, dtype=torch.int32), torch.tensor(kv_len, dtype=torch.int32), shares, free,
             torch.tensor([count], dtype=torch.int32)]
    s.before = torch.cat(parts).to(DEV)
    s.now = s.before.clone()
    s.cuts = _starts([x.numel() for x in parts])
    s.width = width
    s.forks = len(p["forks"])
    s.src = torch.empty((s.forks if case["kind"] == "fork" else s.num_blocks // 2,), dtype=torch.int32, device=DEV)
    s.dst = torch.empty_like(s.src)
    s.status = torch.empty((1,), dtype=torch.int32, device=DEV)
    if case["kind"] == "fork":
        s.parent, s.child = _int32([where[a] for a, _, _ in p["forks"]]), _int32([where[b] for _, b, _ in p["forks"]])
        s.length = _int32([n for _, _, n in p["forks"]])
    s.remap = torch.empty((s.num_blocks,), dtype=torch.int32, device=DEV) if case["kind"] == "compact" else None
    s.moves = torch.empty((1,), dtype=torch.int32, device=DEV)
    shape = (s.num_blocks, case["hkv"], BLOCK, case["head_dim"])
    s.layers = []
    for _ in range(case["layers"]):
        k, ks = _cache_values(shape, case["kv"], gen)
        v, vs = _cache_values(shape, case["kv"], gen)
        s.layers.append((k, v, ks, vs))


def _books(s, flat):
    parts = [flat[a:b] for a, b in zip(s.cuts, s.cuts[1:])]
    return dict(zip(("table", "held", "kv_len", "shares", "free_ids", "free_count"), [parts[0].view(s.batch, s.width)] + parts[1:]))


def _handles_blocks(s, binding):
    case, k = s.case, _books(s, s.now)
    s.d = dict(batch=s.batch, max_blocks_per_seq=s.width, block_table=k["table"], kv_len=k["kv_len"], held=k["held"], shares=k["shares"],
               num_blocks=s.num_blocks, free_ids=k["free_ids"], free_count=k["free_count"])
    s.ws = binding.alloc_block_share_workspace(s.d, DEV, num_forks=s.forks)
    s.handle = binding.cache_layers([dict(num_blocks=s.num_blocks, block_size=BLOCK, num_kv_heads=case["hkv"], head_dim=case["head_dim"],
                                          kv_dtype=case["kv"], k_cache=a, v_cache=b, k_scale=c, v_scale=d) for a, b, c, d in s.layers])


_INPUTS = {"attn": _inputs_attn, "verify": _inputs_verify, "fork": _inputs_blocks, "release": _inputs_blocks, "compact": _inputs_blocks}


def _inputs(case, seed):
    s = _State()
    s.case = case
    _INPUTS[case["kind"]](s, case, seed, _gen(seed))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:     # the descriptions of the batch that the calls take, outputs and workspaces
        from paper_2604_09562_amd import binding
        {"attn": _handles_attn, "verify": _handles_verify}.get(case["kind"], _handles_blocks)(s, binding)
    return s


# ---------------------------------------------------------------------------------------------------
# one pass, in plain operations
# ---------------------------------------------------------------------------------------------------
def _seen(s, L):
    """[batch, max_q, L]: whether a row sees a position."""
    i = torch.arange(s.max_q, device=DEV)
    pos = torch.arange(L, device=DEV)
    q_len = s.q_indptr[1:] - s.q_indptr[:-1]
    row = (s.q_indptr[:-1, None] + i).clamp(max=s.rows - 1).long()
    bits = (s.mask[row][..., (i // 32)] >> (i % 32)) & 1                          # [B, max_q, max_q]
    ctx = (s.kv_len - q_len).long()
    node = (pos - ctx[:, None])                                                    # [B, L]
    inside = (node >= 0) & (node < q_len[:, None])
    picked = bits.gather(2, node.clamp(0, s.max_q - 1)[:, None, :].expand(-1, s.max_q, -1)) > 0
    return (node < 0)[:, None, :] | (inside[:, None, :] & picked), row, i < q_len[:, None]


def _plain_attn(s):
    """All requests side by side, padded to the widest tree and the longest cache."""
    case = s.case
    B, hq, hkv, d = s.batch, case["hq"], case["hkv"], case["head_dim"]
    g, L = hq // hkv, s.table.shape[1] * BLOCK
    ids = s.table.clamp(min=0).long()
    k, v = _at(s.k, ids).float(), _at(s.v, ids).float()                            # [B, blocks, hkv, 16, d]
    if s.k_scale is not None:
        k, v = k * s.k_scale[ids][..., None, None], v * s.v_scale[ids][..., None, None]
    pos = torch.arange(L, device=DEV)
    v = v.transpose(1, 2).reshape(B, hkv, L, d)
    v = torch.where((pos < s.kv_len[:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    k = k.permute(0, 2, 4, 1, 3).reshape(B, hkv, d, L)
    seen, row, there = _seen(s, L)
    q = s.q[row].float().view(B, s.max_q, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, s.max_q * g, d)
    x = torch.matmul(q, k) * s.scale
    x = x.view(B, hkv, s.max_q, g, L).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, s.max_q * g, L), v).view(B, hkv, s.max_q, g, d) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    out = o.permute(0, 2, 1, 3, 4)[there].reshape(s.rows, hq, d).to(s.q.dtype)       # rows in order: requests, then their nodes
    return {"out": out, "lse": lse.permute(0, 2, 1, 3)[there].reshape(s.rows, hq)}


def _plain_verify(s):
    case = s.case
    B, V = s.batch, case["vocab"]
    first, q_len = s.q_indptr[:-1].long(), (s.q_indptr[1:] - s.q_indptr[:-1]).long()
    node = torch.arange(s.max_q, device=DEV)
    row = (first[:, None] + node).clamp(max=s.rows - 1)                               # [B, max_q]
    parent, token = s.parent[row].long(), s.tokens[row].long()
    there = node < q_len[:, None]
    cur = torch.zeros((B,), dtype=torch.int64, device=DEV)
    live = torch.ones((B,), dtype=torch.bool, device=DEV)
    n = torch.zeros((B,), dtype=torch.int32, device=DEV)
    out = torch.full((B, MAX_DEPTH + 1), -1, dtype=torch.int32, device=DEV)
    nodes = torch.full((B, MAX_DEPTH), -1, dtype=torch.int32, device=DEV)
    logp = torch.zeros((B, MAX_DEPTH + 1), device=DEV)
    for step in range(s.depth + 1):
        y, lp = _draw_tokens(s.logits[first + cur, :V], case["temperature"], s.u[first + cur])
        logp[:, step] = torch.where(live, lp, logp[:, step])
        out[:, step] = torch.where(live, y.to(torch.int32), out[:, step])
        if step == s.depth:
            break
        match = there & (node > cur[:, None]) & (parent == cur[:, None]) & (token == y[:, None])
        live = live & match.any(1)
        cur = torch.where(live, match.int().argmax(1), cur)
        nodes[:, step] = torch.where(live, cur.to(torch.int32), nodes[:, step])
        n += live
    return {"accepted_len": n, "out_tokens": out, "accepted_nodes": nodes, "logprobs": logp}


def _raw(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_fork(s):
    k = {name: x.clone() for name, x in _books(s, s.before).items()}
    parent, child, length = s.parent.long(), s.child.long(), s.length
    count = k["free_count"]
    j = torch.arange(s.width, device=DEV)
    whole, part = length // BLOCK, length % BLOCK != 0
    rows = k["table"][parent]
    shared = j < whole[:, None]
    k["shares"].scatter_add_(0, rows.clamp(min=0).view(-1).long(), shared.view(-1).to(torch.int32))
    rank = part.to(torch.int32).cumsum(0, dtype=torch.int32)
    fresh = k["free_ids"][(count - rank).clamp(min=0).long()]
    last = rows.gather(1, whole.clamp(max=s.width - 1)[:, None].long())[:, 0]
    here = (j == whole[:, None]) & part[:, None]
    k["table"][child] = torch.where(shared, rows, torch.where(here, fresh[:, None], k["table"][child]))
    k["held"][child] = (length + BLOCK - 1) // BLOCK
    k["kv_len"][child] = length
    k["free_count"] = count - rank[-1:]
    src, dst = torch.where(part, last, -1), torch.where(part, fresh, -1)
    a, b = torch.where(part, src, rows[:, 0]).long(), torch.where(part, dst, rows[:, 0]).long()     # nothing to copy: a block onto itself
    for layer in s.layers:
        for x in layer:
            if x is not None:
                _raw(x)[b] = _raw(x)[a]
    return dict(k, status=torch.zeros((1,), dtype=torch.int32, device=DEV), src=src, dst=dst, layers=[x for l in s.layers for x in l if x is not None])


def _plain_release(s):
    k = {name: x.clone() for name, x in _books(s, s.before).items()}
    need = (k["kv_len"] + BLOCK - 1) // BLOCK
    j = torch.arange(s.width, device=DEV)
    given = ((j >= need[:, None]) & (j < k["held"][:, None])).view(-1)
    N = s.num_blocks
    at = torch.arange(given.numel(), device=DEV)
    ids = torch.where(given, k["table"].view(-1).long(), N + at)                   # (what is kept: a place of its own behind the blocks)
    times = torch.zeros((N + at.numel(),), dtype=torch.int32, device=DEV).scatter_add_(0, ids, given.to(torch.int32))
    last = torch.full((N + at.numel(),), -1, dtype=torch.int64, device=DEV).scatter_reduce_(0, ids, at, "amax")
    gone = torch.cat([times[:N] > k["shares"], given.new_zeros(at.numel())])
    free = given & (last[ids] == at) & gone[ids]
    place = torch.where(free, k["free_count"] + free.cumsum(0) - 1, N + at)
    pad = torch.cat([k["free_ids"], k["free_ids"].new_zeros(at.numel())]).scatter_(0, place, k["table"].view(-1))
    return dict(k, held=torch.minimum(k["held"], need), shares=(k["shares"] - times[:N]).clamp(min=0), free_ids=pad[:N],
                free_count=k["free_count"] + free.sum().to(torch.int32), status=torch.zeros((1,), dtype=torch.int32, device=DEV))


def _plain_compact(s):
    k = {name: x.clone() for name, x in _books(s, s.before).items()}
    N, count = s.num_blocks, k["free_count"].long()
    i = torch.arange(N, device=DEV)
    free = torch.zeros((N + 1,), dtype=torch.bool, device=DEV)
    free[torch.where(i < count, k["free_ids"].long(), N)] = True
    free = free[:-1]
    used = N - count
    hole, mover = free & (i < used), ~free & (i >= used)
    half = N // 2
    dst = torch.full((half + 1,), -1, dtype=torch.int64, device=DEV).scatter_(0, torch.where(hole, hole.cumsum(0) - 1, half), i)[:half]
    src = torch.full((half + 1,), -1, dtype=torch.int64, device=DEV).scatter_(0, torch.where(mover, mover.cumsum(0) - 1, half), i)[:half]
    moves = mover.sum()
    there = torch.arange(half, device=DEV) < moves
    src, dst = torch.where(there, src, -1), torch.where(there, dst, -1)
    remap = torch.cat([i, i.new_zeros(1)]).scatter_(0, torch.where(there, src, N), dst)[:-1]
    origin = torch.cat([i, i.new_zeros(1)]).scatter_(0, torch.where(there, dst, N), src)[:-1]
    j = torch.arange(s.width, device=DEV)
    k["table"] = torch.where(j < k["held"][:, None], remap[k["table"].clamp(min=0).long()].to(torch.int32), k["table"])
    k["shares"] = torch.where(i < used, k["shares"][origin], torch.zeros_like(k["shares"]))
    k["free_ids"] = torch.where(i < count, N - 1 - i, k["free_ids"].long()).to(torch.int32)
    for layer in s.layers:
        for x in layer:
            if x is not None:
                _raw(x).copy_(_raw(x)[origin])
    as32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(k, status=torch.zeros((1,), dtype=torch.int32, device=DEV), src=as32(src), dst=as32(dst), remap=as32(remap), moves=as32(moves).view(1),
                layers=[x for l in s.layers for x in l if x is not None])


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"attn": _plain_attn, "verify": _plain_verify, "fork": _plain_fork, "release": _plain_release, "compact": _plain_compact}[kind](s)
    from paper_2604_09562_amd import binding
    if kind == "attn":
        binding.ss_tree_attn(s.d, s.out, s.lse, s.ws, max_q_len=s.max_q)
        return {"out": s.out if s.out.dtype == torch.float32 else s.out.view(torch.bfloat16), "lse": s.lse}
    if kind == "verify":
        binding.ss_tree_verify(s.d, s.n, s.out, s.nodes, s.logp, s.ws, max_depth=s.depth)
        return {"accepted_len": s.n, "out_tokens": s.out, "accepted_nodes": s.nodes, "logprobs": s.logp}
    s.now.copy_(s.before)
    books = dict(_books(s, s.now), status=s.status)
    if kind == "release":
        binding.ss_block_release(s.d, s.status, s.ws)
        return books
    layers = [x for l in s.layers for x in l if x is not None]
    if kind == "fork":
        binding.ss_block_fork(s.d, s.parent, s.child, s.length, s.src, s.dst, s.status, s.ws)
        binding.ss_block_copy(s.handle, s.src, s.dst)
        return dict(books, src=s.src, dst=s.dst, layers=layers)
    binding.ss_block_compact(s.d, s.remap, s.src, s.dst, s.moves, s.status, s.ws)
    binding.ss_block_copy(s.handle, s.src, s.dst, s.moves)
    return dict(books, src=s.src, dst=s.dst, remap=s.remap, moves=s.moves, layers=layers)


# ---------------------------------------------------------------------------------------------------
# the definitions in 64 bits, one request (and one head) after the other
# ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "attn":
        return _exact_attn(case, _inputs(case, seed))
    if case["kind"] == "verify":
        return {"accepted_len": None, "out_tokens": None, "accepted_nodes": None, "logprobs": _exact_logprobs(case, _inputs(case, seed))}
    return None     # whole numbers and copies


def _exact_logprobs(case, s):
    out = torch.zeros((s.batch, MAX_DEPTH + 1), dtype=torch.float64)
    if case["temperature"] == 0.0:
        return out.to(DEV)
    ends, parent, tokens, u = s.q_indptr.tolist(), s.parent.tolist(), s.tokens.tolist(), s.u.tolist()
    for b in range(s.batch):
        r0, r1 = ends[b], ends[b + 1]
        cur = 0
        for step in range(case["depth"] + 1):
            p = torch.softmax(s.logits[r0 + cur, :case["vocab"]].double() / case["temperature"], 0)
            y = int(torch.searchsorted(p.cumsum(0), torch.tensor([u[r0 + cur]], dtype=torch.float64, device=DEV), right=True).clamp(max=case["vocab"] - 1))
            out[b, step] = p[y].log()
            below = [c for c in range(cur + 1, r1 - r0) if parent[r0 + c] == cur and tokens[r0 + c] == y]
            if not below:
                break
            cur = below[0]
    return out.to(DEV)


def _exact_attn(case, s):
    hq, hkv, d = case["hq"], case["hkv"], case["head_dim"]
    g = hq // hkv
    out = torch.empty((s.rows, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((s.rows, hq), dtype=torch.float64, device=DEV)
    ends, lens, words = s.q_indptr.tolist(), s.kv_len.tolist(), s.mask.tolist()
    for b, m in enumerate(lens):
        r0, r1 = ends[b], ends[b + 1]
        n = r1 - r0
        ids = s.table[b, :_blocks(m)].long()
        sees = torch.ones((n, m), dtype=torch.bool)
        sees[:, m - n:] = torch.tensor([[words[r0 + i][j // 32] >> (j % 32) & 1 for j in range(n)] for i in range(n)], dtype=torch.bool)
        sees = sees.to(DEV)[:, None]
        for h in range(hkv):
            k, v = _at(s.k[:, h], ids).double(), _at(s.v[:, h], ids).double()
            if s.k_scale is not None:
                k, v = k * s.k_scale[ids, h].double()[:, None, None], v * s.v_scale[ids, h].double()[:, None, None]
            k, v = k.reshape(-1, d)[:m], v.reshape(-1, d)[:m]
            q = s.q[r0:r1, h * g:(h + 1) * g].double().reshape(-1, d)
            x = torch.where(sees, (q @ k.T.contiguous()).view(n, g, m) / math.sqrt(d), -math.inf)
            z = torch.logsumexp(x, -1)
            out[r0:r1, h * g:(h + 1) * g] = ((x - z[..., None]).exp().view(-1, m) @ v).view(n, g, d)
            lse[r0:r1, h * g:(h + 1) * g] = z
    return {"out": out, "lse": lse}
