"""ss_tree_verify at infinite temperatures: every token that is not masked is alike, whatever its logit, in both forms of the call."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from .prefill_ref import DEV
from .test_gpu_tree_verify import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,max_depth,rounds", [(12, 5003, 0, False), (600, 40000, 1, False), (600, 40000, 1, True)])
def test_every_token_that_is_not_masked_is_alike(rows, vocab, max_depth, rounds, dtype):
    rng = np.random.default_rng(rows)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    low, high = torch.finfo(kind).min, torch.finfo(kind).max
    x = torch.from_numpy(rng.standard_normal((rows, vocab), dtype=np.float32) * 3)
    x[:, ::3] = low                      # a common fill value, near ordinary logits
    x[:, 1::17] = -1e36
    x[1::4, 5::31] = high                # and as far above them
    masked = torch.from_numpy(rng.random((rows, vocab), dtype=np.float32) < 0.2)
    masked[2] = False
    masked[3, :-1] = True
    masked[3, -1] = False
    x = torch.where(masked, torch.from_numpy(rng.choice(np.float32([-np.inf, np.nan]), vocab)), x)
    left = [np.flatnonzero(~m) for m in masked.numpy()]
    # the middle of a token's share of the uniforms: at most 40000 shares are 2^-15.3 wide, a float below 1 is 2^-25 off
    place = [int(rng.integers(0, len(y))) for y in left]
    u = np.array([(p + 0.5) / len(y) for p, y in zip(place, left)], np.float32)
    indptr = np.arange(rows + 1, dtype=np.int32)
    h = dict(batch=rows, vocab=vocab, row_stride=(vocab + 7) // 8 * 8, logit_dtype=dtype, total_rows=rows, q_indptr=indptr, tree_parent=np.full(rows, -1, np.int32),
             node_tokens=np.zeros(rows, np.int32), uniforms=u, temp=np.full(rows, np.inf, np.float32),
             logits=torch.nn.functional.pad(x, (0, -vocab % 8)).to(kind))
    for scalar in (False, True):
        d = device(h, scalar)
        n, out, nodes, lp, ws = binding.alloc_tree_verify_outputs(d, DEV)
        if rounds:      # in the room that they need the rows are taken in rounds
            ws = ws[:binding.lib().ss_tree_verify_workspace(rows, 0, vocab)]
        binding.ss_tree_verify(d, n, out, nodes, lp, ws, max_depth=max_depth)
        torch.cuda.synchronize()
        assert not n.any()
        assert np.array_equal(out[:, 0].cpu().numpy(), [y[p] for p, y in zip(place, left)])
        want = -np.log([len(y) for y in left])
        off = np.abs(lp[:, 0].cpu().numpy().astype(np.float64) - want)
        assert (off <= 2.0 ** -24 * np.abs(want) * 1.01 + 1e-12).all(), off.max()      # (one rounding to 32 bits; sums of ones are exact)
