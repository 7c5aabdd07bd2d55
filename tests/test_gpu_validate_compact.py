"""Option "validate" and ss_kv_compact: what is inconsistent is named; requests without new tokens and rows behind the last request are none of that."""
import numpy as np
import pytest
import torch

from paper_2604_09562_amd import binding

from .test_gpu_path_compaction import batch, check, i32, moved

pytestmark = pytest.mark.gpu

LENGTHS = [(40, 100), (0, 90), (50, 50), (0, 0), (1, 1), (30, 64)]


@pytest.fixture()
def validating():
    binding.ss_set_option("validate", 1)
    yield
    binding.ss_set_option("validate", 0)


def test_consistent_batches_pass(validating):
    d, nodes, n_acc = batch("bf16", LENGTHS, 1)
    want = moved(d, nodes, n_acc, LENGTHS)
    binding.ss_kv_compact(dict(d, total_rows=d["total_rows"] + 7), i32(nodes), i32(n_acc))
    torch.cuda.synchronize()
    check(d, want)


@pytest.mark.parametrize("b,kv_len,text", [(2, 49, "request 2 has kv_len 49 but 50 query rows"), (0, 39, "request 0 has kv_len 39 but 40"), (4, 0, "request 4 has kv_len 0 but 1"),
                                           (5, -1, "request 5 has kv_len -1"), (1, -3, "request 1 has kv_len -3"), (5, 10 ** 6, "request 5 .* blocks")])
def test_lengths_that_cannot_be_are_named(validating, b, kv_len, text):
    d, nodes, n_acc = batch("bf16", LENGTHS, 2)
    before = [d["k_cache"].clone(), d["v_cache"].clone()]
    d["kv_len"][b] = kv_len
    with pytest.raises(binding.SpecVerifyError, match="ss_kv_compact: " + text):
        binding.ss_kv_compact(d, i32(nodes), i32(n_acc))
    torch.cuda.synchronize()
    check(d, before)
