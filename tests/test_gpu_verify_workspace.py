"""ss_tree_verify in workspaces of other sizes than its own: one for a larger step serves, and what is left free of it stays as it was."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from . import share_ref as ref
from .prefill_ref import DEV
from .test_gpu_tree_verify import batch, device

pytestmark = pytest.mark.gpu


def sized(B, rows, vocab):
    return binding.lib().ss_tree_verify_workspace(B, rows, vocab)


def run(h, n, max_depth=0):
    """The call in a workspace of n bytes, in front of others that have to stay as they are."""
    d = device(h)
    out = binding.alloc_tree_verify_outputs(d, DEV)[:4]
    room = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    binding.ss_tree_verify(d, *out, room[:n], max_depth=max_depth)
    torch.cuda.synchronize()
    assert (room[n:] == 0xA5).all()
    w = ref.verify(h["exact"], h["q_indptr"], h["total_rows"], h["tree_parent"], h["node_tokens"], h["uniforms"], h["temp"], max_depth or 20)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out[:3], w[:3]))


@pytest.mark.parametrize("nodes,vocab,bounds", [([25], 32000, (1, 3300)), ([5, 0, 40, 1], 128256, (64, 4096)), ([12] * 64, 5000, (64, 1 << 20)), ([900], 100, (1, 1 << 22)),
                                                ([3000, 9], 40, (4, 1 << 26))])
def test_one_of_a_larger_step(nodes, vocab, bounds):
    run(batch(nodes, vocab, seed=len(nodes)), sized(*bounds, vocab))


def test_too_little_room_is_refused():
    h = batch([25, 9], 3000, seed=4)
    d = device(h)
    out = binding.alloc_tree_verify_outputs(d, DEV)[:4]
    least = sized(2, 0, 3000)
    run(h, least)        # a row's room for each round is enough: the rows are taken in rounds
    with pytest.raises(binding.SpecVerifyError, match="needed"):
        binding.ss_tree_verify(d, *out, torch.empty(least - 1, dtype=torch.uint8, device=DEV))
