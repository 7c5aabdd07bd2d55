"""Plain references, in 64 bits or whole numbers, of the calls that fill the paged cache, and the batches the tests give them."""
import numpy as np
import torch

BLOCK = 16
DEV = "cuda:0"
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step of the type, relative
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def blocks(n):
    return -(-n // BLOCK)


# ---------------------------------------------------------------------------------------------------
# block tables and slot maps
# ---------------------------------------------------------------------------------------------------
def block_map(table, held, ids, count, kv_len, q_indptr, total_rows, num_blocks):
    """The definition with a list for the free blocks: (table, held, free list padded as given, count, slots, positions, status)."""
    B, width = table.shape
    table, held, ids = table.copy(), held.copy(), ids.copy()
    slots, positions = np.full(total_rows, -1, np.int32), np.full(total_rows, -1, np.int32)
    for b in range(B):
        q0, q1, n, h = int(q_indptr[b]), int(q_indptr[b + 1]), int(kv_len[b]), int(held[b])
        if q0 < 0 or q1 < q0 or q1 > total_rows or (b == 0 and q0 != 0) or n < q1 - q0 or blocks(n) > width or not 0 <= h <= width:
            return table, held, ids, count, slots, positions, -1 - b
    need = [blocks(int(n)) for n in kv_len]
    after = count + sum(int(h) for h in held) - sum(need)
    if count < 0 or after > num_blocks:
        return table, held, ids, count, slots, positions, -1 - B
    if after < 0:
        return table, held, ids, count, slots, positions, -after
    free = [int(x) for x in ids[:count]]
    for b in range(B):
        free += [int(table[b, j]) for j in range(need[b], held[b])]
    for b in range(B):
        for j in range(held[b], need[b]):
            table[b, j] = free.pop()
    ids[:len(free)] = free
    held[:] = need
    for b in range(B):
        q0, q1 = int(q_indptr[b]), int(q_indptr[b + 1])
        for r in range(q0, q1):
            pos = int(kv_len[b]) - q1 + r
            positions[r] = pos
            slots[r] = int(table[b, pos // BLOCK]) * BLOCK + pos % BLOCK
    return table, held, ids, len(free), slots, positions, 0


def map_batch(lengths, held, extra_free=7, spare_rows=0, spare_columns=0, seed=0):
    """A batch of (new tokens, cache length) and blocks held: dict of numpy arrays with the state before the call."""
    rng = np.random.default_rng(seed)
    B = len(lengths)
    width = max([blocks(n) for _, n in lengths] + list(held) + [1]) + spare_columns
    grow = sum(max(blocks(n) - h, 0) for (_, n), h in zip(lengths, held))
    total = sum(held) + grow + extra_free
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((B, width), -5, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = perm[at:at + h]
        at += h
    ids = np.full(total, -9, np.int32)
    ids[:total - at] = perm[at:]
    indptr = np.zeros(B + 1, np.int32)
    indptr[1:] = np.cumsum([q for q, _ in lengths])
    return dict(table=table, held=np.array(held, np.int32).reshape(B), ids=ids, count=total - at, kv_len=np.array([n for _, n in lengths], np.int32).reshape(B),
                q_indptr=indptr, total_rows=int(indptr[-1]) + spare_rows, num_blocks=total)


# ---------------------------------------------------------------------------------------------------
# caches
# ---------------------------------------------------------------------------------------------------
def cache_values(shape, dtype, gen, device=DEV):
    """(keys or values in storage format, scales or None)"""
    if dtype != "fp8":
        return torch.randn(shape, generator=gen, device=device).to(TORCH[dtype]), None
    scale = torch.rand(shape[:2], generator=gen, device=device) * 0.09 + 0.01
    x = torch.randn(shape, generator=gen, device=device) / scale[:, :, None, None]
    return x.clamp_(-448.0, 448.0).to(TORCH["fp8"]), scale


def decoded(cache, scale):
    x = cache.cpu().to(torch.float64)
    return x if scale is None else x * scale.cpu().to(torch.float64)[:, :, None, None]


# ---------------------------------------------------------------------------------------------------
# attention of chunks
# ---------------------------------------------------------------------------------------------------
def chunk_batch(lengths, hq, hkv, d, kv="bf16", q="bf16", seed=0, spare_rows=0, spare_columns=0, sharp=2.0, row_pad=0, garbage=True):
    """A batch of (new tokens, cache length): dict as the binding takes it, on the GPU.  What no row may see holds NaN."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    counts = [blocks(n) for _, n in lengths]
    used = sum(counts)
    total = used + 3
    perm = torch.randperm(total, generator=torch.Generator().manual_seed(seed))[:used].to(torch.int32)
    width = max(counts + [1]) + spare_columns
    table = torch.full((len(lengths), width), 0x7FFFFFF0, dtype=torch.int32)    # not to be used
    k, ks = cache_values((total, hkv, BLOCK, d), kv, gen)
    v, vs = cache_values((total, hkv, BLOCK, d), kv, gen)
    live = torch.zeros((total, BLOCK), dtype=torch.bool)
    at = 0
    for b, (_, n) in enumerate(lengths):
        table[b, :counts[b]] = perm[at:at + counts[b]]
        for j in range(counts[b]):
            live[int(perm[at + j]), :min(BLOCK, n - j * BLOCK)] = True
        at += counts[b]
    if garbage:
        dead = (~live).to(DEV)[:, None, :].expand(total, hkv, BLOCK)
        for cache in (k, v):
            raw = cache.view(torch.uint8) if kv == "fp8" else cache
            raw[dead] = 0x7F if kv == "fp8" else float("nan")
    indptr = [0]
    for n, _ in lengths:
        indptr.append(indptr[-1] + n)
    rows = indptr[-1] + spare_rows
    wide = torch.randn((rows, hq * d + row_pad), generator=gen, device=DEV) * sharp
    wide = wide.to(TORCH[q])
    qt = wide[:, :hq * d].unflatten(1, (hq, d))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(batch=len(lengths), num_q_heads=hq, num_kv_heads=hkv, head_dim=d, block_size=BLOCK, num_blocks=total,
                max_blocks_per_seq=width, total_rows=rows, kv_dtype=kv, q_dtype=q, kv_len=i32([n for _, n in lengths]), q_indptr=i32(indptr),
                block_table=table.to(DEV), k_cache=k, v_cache=v, k_scale=ks, v_scale=vs, q=qt, sm_scale=1.0 / d ** 0.5)


def chunk_reference(inp):
    """(out, lse, mean |v| under the weights, largest sum of |q||k| of a row's scores) in 64 bits; rows of no request are NaN."""
    hq, hkv, d = inp["num_q_heads"], inp["num_kv_heads"], inp["head_dim"]
    g = hq // hkv
    rows = inp["total_rows"]
    out = torch.full((rows, hq, d), float("nan"), dtype=torch.float64, device=DEV)
    size = torch.full((rows, hq, d), float("nan"), dtype=torch.float64, device=DEV)
    lse = torch.full((rows, hq), float("nan"), dtype=torch.float64, device=DEV)
    mag = torch.zeros((rows, hq), dtype=torch.float64, device=DEV)
    indptr, lens = inp["q_indptr"].tolist(), inp["kv_len"].tolist()
    for b, n in enumerate(lens):
        r0, r1 = indptr[b], indptr[b + 1]
        if r1 == r0:
            continue
        ids = inp["block_table"][b, :blocks(n)].long()
        for h in range(hkv):
            def gathered(cache, scale):
                raw = cache.view(torch.uint8)[:, h][ids].view(cache.dtype) if cache.dtype == TORCH["fp8"] else cache[:, h][ids]
                x = raw.double()
                if scale is not None:
                    x = x * scale[ids, h].double()[:, None, None]
                return x.reshape(-1, d)[:n]
            k, v = gathered(inp["k_cache"], inp["k_scale"]), gathered(inp["v_cache"], inp["v_scale"])
            q = inp["q"][r0:r1, h * g:(h + 1) * g].double()
            last = torch.arange(r1 - r0, device=DEV) + n - (r1 - r0)
            if n == 0:
                out[r0:r1, h * g:(h + 1) * g], size[r0:r1, h * g:(h + 1) * g] = 0.0, 0.0
                lse[r0:r1, h * g:(h + 1) * g] = -float("inf")
                continue
            seen = (torch.arange(n, device=DEV) <= last[:, None])[:, None]
            kt = k.T.contiguous()
            x = torch.where(seen, (q.reshape(-1, d) @ kt).view(r1 - r0, g, n) * inp["sm_scale"], -float("inf"))
            z = torch.logsumexp(x, -1)
            p = torch.where(seen, (x - torch.where(z.isfinite(), z, torch.zeros_like(z))[..., None]).exp(), 0.0).view(-1, n)
            out[r0:r1, h * g:(h + 1) * g] = (p @ v).view(r1 - r0, g, d)
            size[r0:r1, h * g:(h + 1) * g] = (p @ v.abs()).view(r1 - r0, g, d)
            lse[r0:r1, h * g:(h + 1) * g] = z
            mag[r0:r1, h * g:(h + 1) * g] = ((q.reshape(-1, d).abs() @ kt.abs()).view(r1 - r0, g, n) * seen).amax(-1) * inp["sm_scale"]
    return out, lse, size, mag


def chunk_tolerances(inp, out, lse, size, mag):
    """Bounds on |out - ref| and |lse - ref| by arithmetic.

    A score is a sum of d products in fp32, each product exact or rounded once, and is taken to a power of two with a few more
    roundings: its error is below (d + 8) 2^-24 of the sum of the magnitudes.  An exponential has that as relative error, and 2^-22 of
    its own.  Sums over n keys add n 2^-24 of the sum of the magnitudes.  Weights in bf16 (bf16 queries over bf16 or e4m3
    caches) are off by half a step each; the result by half a step of its type.
    """
    n = float(inp["kv_len"].max())
    score = (inp["head_dim"] + 8) * 2.0 ** -24 * mag
    bf16 = inp["q_dtype"] == "bf16" and inp["kv_dtype"] != "f32"
    each = (2 * score + (2 * n + 16) * 2.0 ** -24 + 2.0 ** -21)[..., None] + (HALF["bf16"] if bf16 else 0.0)
    tol = each * size + HALF[inp["q_dtype"]] * out.abs() * 1.01 + 1e-30
    return tol, score + (n + 16) * 2.0 ** -24 + 2.0 ** -21 + lse.abs() * 2.0 ** -22


def check_chunk(inp, got_out, got_lse, label=""):
    ref, lse, size, mag = chunk_reference(inp)
    tol, ltol = chunk_tolerances(inp, ref, lse, size, mag)
    used = int(inp["q_indptr"][-1])
    out = (got_out if got_out.dtype == torch.float32 else got_out.view(torch.bfloat16)).double()
    off = (out - ref).abs()[:used]
    bad = ~(off <= tol[:used])
    assert not bad.any(), f"{label}: {int(bad.sum())} of {bad.numel()} outputs off, first {bad.nonzero()[0].tolist()}, largest {off.nan_to_num(9e9).max():.3e}"
    none = torch.isinf(lse[:used])
    assert torch.equal(torch.isinf(got_lse[:used]) & (got_lse[:used] < 0), none), f"{label}: rows that see nothing"
    loff = torch.where(none, 0.0, (got_lse.double()[:used] - lse[:used]).abs())
    assert (loff <= ltol[:used]).logical_or(none).all(), f"{label}: lse off by {loff.max():.3e}"
