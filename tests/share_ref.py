"""Plain references, in 64 bits or whole numbers, of the calls for wide draft trees and shared blocks, and the batches the tests give them."""
import math

import numpy as np
import torch

from .prefill_ref import BLOCK, DEV, TORCH, blocks, chunk_batch, chunk_tolerances


# ---------------------------------------------------------------------------------------------------
# trees and their masks
# ---------------------------------------------------------------------------------------------------
def random_tree(n, rng, depth=10 ** 6):
    """Parents of a random tree, -1 for node 0."""
    parent, level = [-1], [0]
    for i in range(1, n):
        p = int(rng.integers(0, i))
        while level[p] >= depth:
            p = int(rng.integers(0, i))
        parent.append(p)
        level.append(level[p] + 1)
    return parent[:n]


def ancestors(parent):
    """bool [n][n]: a node's own place and its ancestors'."""
    n = len(parent)
    sees = np.zeros((n, n), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def pack(sees, words):
    """uint32 words of a bool matrix, least significant bit first."""
    n, m = sees.shape
    wide = np.zeros((n, words * 32), bool)
    wide[:, :m] = sees
    return np.packbits(wide.reshape(n, words, 32), axis=2, bitorder="little").view("<u4").reshape(n, words)


def tree_batch(lengths, hq, hkv, d, pattern="tree", spare_words=0, stray_bits=False, **kw):
    """chunk_batch of (nodes, cache length) with masks: dict as the binding takes it, with the bool matrices in `sees`."""
    inp = chunk_batch(lengths, hq, hkv, d, **kw)
    rng = np.random.default_rng(kw.get("seed", 0) + 17)
    words = max([1] + [-(-n // 32) for n, _ in lengths]) + spare_words
    mask = rng.integers(0, 2 ** 32, (inp["total_rows"], words), dtype=np.uint64).astype(np.uint32)
    sees, at = [], 0
    for n, _ in lengths:
        if pattern == "tree":
            s = ancestors(random_tree(n, rng))
        elif pattern == "chain":
            s = np.tril(np.ones((n, n), bool))
        elif pattern == "all":
            s = np.ones((n, n), bool)
        elif pattern == "none":
            s = np.zeros((n, n), bool)
        else:
            s = rng.random((n, n)) < 0.3
        w = pack(s, words)
        if stray_bits and n:   # behind the last node: not to be looked at
            w |= pack(np.pad(np.zeros((n, n), bool), ((0, 0), (0, words * 32 - n)), constant_values=True), words)
        mask[at:at + n] = w
        sees.append(s)
        at += n
    return dict(inp, node_mask=torch.from_numpy(mask.view(np.int32)).to(DEV), sees=sees)


def gathered(inp, b, h, n):
    """(keys, values) [n][d] of a request's KV head in 64 bits."""
    ids = inp["block_table"][b, :blocks(n)].long()
    out = []
    for cache, scale in ((inp["k_cache"], inp["k_scale"]), (inp["v_cache"], inp["v_scale"])):
        x = (cache.view(torch.uint8)[:, h][ids].view(cache.dtype) if cache.dtype == TORCH["fp8"] else cache[:, h][ids]).double()
        if scale is not None:
            x = x * scale[ids, h].double()[:, None, None]
        out.append(x.reshape(-1, inp["head_dim"])[:n])
    return out


def tree_reference(inp):
    """(out, lse, mean |v| under the weights, largest sum of |q||k| of a row's scores) in 64 bits; rows of no request are NaN."""
    hq, hkv, d = inp["num_q_heads"], inp["num_kv_heads"], inp["head_dim"]
    g, rows = hq // hkv, inp["total_rows"]
    out = torch.full((rows, hq, d), float("nan"), dtype=torch.float64, device=DEV)
    size = out.clone()
    lse = torch.full((rows, hq), float("nan"), dtype=torch.float64, device=DEV)
    mag = torch.zeros((rows, hq), dtype=torch.float64, device=DEV)
    indptr, lens = inp["q_indptr"].tolist(), inp["kv_len"].tolist()
    for b, n in enumerate(lens):
        r0, r1 = indptr[b], indptr[b + 1]
        q_len = r1 - r0
        if q_len == 0:
            continue
        seen = torch.ones((q_len, n), dtype=torch.bool)
        for t in range(max(n - q_len, 0), n):
            seen[:, t] = torch.from_numpy(inp["sees"][b][:, t - (n - q_len)].copy())
        seen = seen.to(DEV)[:, None]
        for h in range(hkv):
            at = (slice(r0, r1), slice(h * g, (h + 1) * g))
            q = inp["q"][at].double().reshape(-1, d)
            if n == 0:
                out[at], size[at], lse[at] = 0.0, 0.0, -math.inf
                continue
            k, v = gathered(inp, b, h, n)
            kt = k.T.contiguous()
            x = torch.where(seen, (q @ kt).view(q_len, g, n) * inp["sm_scale"], -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.where(seen, (x - torch.where(z.isfinite(), z, torch.zeros_like(z))[..., None]).exp(), 0.0)
            for r in range(q_len):      # (row by row, so that what a row does not see stays out of its sum whatever it is)
                s = seen[r, 0]
                out[r0 + r, h * g:(h + 1) * g] = p[r][:, s] @ v[s]
                size[r0 + r, h * g:(h + 1) * g] = p[r][:, s] @ v[s].abs()
            lse[at] = z
            mag[at] = torch.where(seen, (q.abs() @ kt.abs()).view(q_len, g, n), 0.0).amax(-1) * inp["sm_scale"]
    return out, lse, size, mag


def check_tree(inp, got_out, got_lse, label="", rows=None):
    """Outputs within the bounds of chunk_tolerances; rows: which of them."""
    ref, lse, size, mag = tree_reference(inp)
    tol, ltol = chunk_tolerances(inp, ref, lse, size, mag)
    used = torch.arange(int(inp["q_indptr"][-1]), device=DEV) if rows is None else rows
    out = (got_out if got_out.dtype == torch.float32 else got_out.view(torch.bfloat16)).double()
    off = (out - ref).abs()[used]
    bad = ~(off <= tol[used])
    assert not bad.any(), f"{label}: {int(bad.sum())} of {bad.numel()} outputs off, first {bad.nonzero()[0].tolist()}, largest {off.nan_to_num(9e9).max():.3e}"
    none = torch.isinf(lse[used])
    assert torch.equal(torch.isinf(got_lse[used]) & (got_lse[used] < 0), none), f"{label}: rows that see nothing"
    loff = torch.where(none, 0.0, (got_lse.double()[used] - lse[used]).abs())
    assert (loff <= ltol[used]).logical_or(none).all(), f"{label}: lse off by {loff.max():.3e}"


# ---------------------------------------------------------------------------------------------------
# the walk through a tree by the target's own draws
# ---------------------------------------------------------------------------------------------------
def draw(row, temperature, u):
    """(token, ln p) of one row of logits (float64)."""
    x = np.where(np.isnan(row), -np.inf, row)
    m = x.max()
    if m == -np.inf:
        return 0, 0.0
    if not temperature > 0 or m == np.inf:
        return int(np.argmax(x)), 0.0
    with np.errstate(over="ignore", under="ignore"):
        e = np.exp((x - m) / np.float64(temperature))
    c = np.cumsum(e)
    over = np.nonzero((c > float(u) * c[-1]) & (e > 0))[0]
    y = int(over[0]) if len(over) else int(np.nonzero(e > 0)[0][-1])
    return y, (x[y] - m) / np.float64(temperature) - math.log(c[-1])


def verify(logits, q_indptr, total_rows, parent, tokens, u, temperature, max_depth, width=21):
    """(accepted_len, out_tokens, accepted_nodes, logprobs) by the definition; logits float64 [rows][vocab]."""
    B = len(q_indptr) - 1
    n = np.zeros(B, np.int32)
    out, nodes, lp = np.full((B, width), -1, np.int32), np.full((B, width - 1), -1, np.int32), np.zeros((B, width))
    for b in range(B):
        r0, r1 = int(q_indptr[b]), int(q_indptr[b + 1])
        if not (0 <= r0 < r1 <= total_rows):
            continue
        cur = 0
        while True:
            y, out_lp = draw(logits[r0 + cur], temperature[b], u[r0 + cur])
            out[b, n[b]], lp[b, n[b]] = y, out_lp
            if n[b] == max_depth:
                break
            below = [c for c in range(cur + 1, r1 - r0) if parent[r0 + c] == cur and tokens[r0 + c] == y]
            if not below:
                break
            cur = below[0]
            nodes[b, n[b]] = cur
            n[b] += 1
    return n, out, nodes, lp


# ---------------------------------------------------------------------------------------------------
# books of shared blocks
# ---------------------------------------------------------------------------------------------------
def random_books(rng, batch, width, spare, families=3, empty=2):
    """Requests that share blocks as forks leave them: dict of numpy arrays.  `empty` rows at random places hold nothing."""
    rows, shares, used = [], [], 0
    for b in range(batch - empty):
        room = width * BLOCK
        if rows and b % families:
            base, n0 = rows[int(rng.integers(0, len(rows)))]
            at = int(rng.integers(0, n0 + 1))
            ids = base[:at // BLOCK]
            for x in ids:
                shares[x] += 1
            n = min(at + int(rng.integers(0, 70)), room)
        else:
            ids, n = [], int(rng.integers(1, room + 1))
        fresh = blocks(n) - len(ids)
        ids = ids + list(range(used, used + fresh))
        used += fresh
        shares += [0] * fresh
        rows.append((ids, n))
    total = used + spare
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((batch, width), -3, np.int32)
    held, kv_len = np.zeros(batch, np.int32), np.zeros(batch, np.int32)
    for (ids, n), b in zip(rows, rng.permutation(batch)):
        table[b, :len(ids)] = perm[ids]
        held[b], kv_len[b] = len(ids), n
    sh = np.zeros(total, np.int32)
    sh[perm[:used]] = shares
    free = np.full(total, -9, np.int32)
    free[:spare] = perm[used:]
    return dict(table=table, held=held, kv_len=kv_len, shares=sh, free=free, count=spare, num_blocks=total)


def check_books(k):
    """Every block's holders are what shares and the free list say."""
    holders = np.zeros(k["num_blocks"], int)
    for b in range(len(k["held"])):
        for x in k["table"][b, :k["held"][b]]:
            holders[x] += 1
    free = k["free"][:k["count"]]
    assert len(set(free.tolist())) == k["count"] and (holders[free] == 0).all() and (holders > 0).sum() + k["count"] == k["num_blocks"]
    assert np.array_equal(np.maximum(holders - 1, 0), k["shares"])


def copy_of(k):
    return {name: (x.copy() if isinstance(x, np.ndarray) else x) for name, x in k.items()}


def fork(k, parent, child, length):
    """One fork after the other: (books, copy_src, copy_dst, status)."""
    n, width = len(parent), k["table"].shape[1]
    B = len(k["held"])
    none = np.full(n, -1, np.int32)
    children = [int(c) for p, c in zip(parent, child) if p >= 0]
    seen = set()
    for i in range(n):
        p, c = int(parent[i]), int(child[i])
        if p < 0:
            continue
        ok = p < B and 0 <= c < B and c not in seen and p not in children
        if ok:
            m = int(k["kv_len"][p]) if length is None else int(length[i])
            ok = k["held"][c] == 0 and 0 <= m <= k["kv_len"][p] and 0 <= k["held"][p] and blocks(m) <= min(k["held"][p], width)
        if not ok:
            return k, none, none.copy(), -1 - i
        seen.add(c)
    if not 0 <= k["count"] <= k["num_blocks"]:
        return k, none, none.copy(), -1 - n
    lens = [0 if parent[i] < 0 else int(k["kv_len"][parent[i]] if length is None else length[i]) for i in range(n)]
    missing = sum(m % BLOCK != 0 for m in lens) - k["count"]
    if missing > 0:
        return k, none, none.copy(), missing
    k, src, dst = copy_of(k), none, none.copy()
    for i in range(n):
        p, c, m = int(parent[i]), int(child[i]), lens[i]
        if p < 0:
            continue
        for j in range(m // BLOCK):
            k["table"][c, j] = k["table"][p, j]
            k["shares"][k["table"][p, j]] += 1
        if m % BLOCK:
            k["count"] -= 1
            src[i], dst[i] = k["table"][p, m // BLOCK], k["free"][k["count"]]
            k["table"][c, m // BLOCK] = dst[i]
        k["held"][c], k["kv_len"][c] = blocks(m), m
    return k, src, dst, 0


def release(k):
    """One block after the other: (books, status)."""
    B, width = k["table"].shape
    for b in range(B):
        if k["kv_len"][b] < 0 or not 0 <= k["held"][b] <= width:
            return k, -1 - b
    if not 0 <= k["count"] <= k["num_blocks"]:
        return k, -1 - B
    k = copy_of(k)
    given = [int(k["table"][b, j]) for b in range(B) for j in range(blocks(int(k["kv_len"][b])), k["held"][b])]
    given = [x for x in given if 0 <= x < k["num_blocks"]]
    for r, x in enumerate(given):
        k["shares"][x] -= 1
    for r, x in enumerate(given):
        if k["shares"][x] < 0 and x not in given[r + 1:]:
            k["free"][k["count"]] = x
            k["count"] += 1
    k["shares"] = np.maximum(k["shares"], 0)
    k["held"] = np.minimum(k["held"], [blocks(int(n)) for n in k["kv_len"]]).astype(np.int32)
    return k, 0


def compact(k):
    """(books, remap, copy_src, copy_dst, moves, status)."""
    N, (B, width) = k["num_blocks"], k["table"].shape
    none = np.full(N // 2, -1, np.int32)
    status = 0
    free = k["free"][:max(min(k["count"], N), 0)]
    if not 0 <= k["count"] <= N or any(not 0 <= x < N for x in free) or len(set(free.tolist())) != len(free):
        status = -1 - B
    for b in reversed(range(B)):
        if not 0 <= k["held"][b] <= width:
            status = -1 - b
    if status:
        return k, np.arange(N, dtype=np.int32), none, none.copy(), 0, status
    k, used = copy_of(k), N - k["count"]
    is_free = set(free.tolist())
    holes = [i for i in range(used) if i in is_free]
    movers = [i for i in range(used, N) if i not in is_free]
    remap, src, dst = np.arange(N, dtype=np.int32), none, none.copy()
    for r, (i, j) in enumerate(zip(movers, holes)):
        remap[i], src[r], dst[r] = j, i, j
        k["shares"][j], k["shares"][i] = k["shares"][i], 0
    for b in range(B):
        for j in range(k["held"][b]):
            if 0 <= k["table"][b, j] < N:
                k["table"][b, j] = remap[k["table"][b, j]]
    k["free"][:k["count"]] = N - 1 - np.arange(k["count"])
    return k, remap, src, dst, len(movers), 0
