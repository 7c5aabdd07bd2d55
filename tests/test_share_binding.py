"""The books of shared blocks are looked at in every call of the binding, not only where a workspace is allocated: no GPU needed."""
import pytest
import torch

from paper_2604_09562_amd import binding


class OnCard(torch.Tensor):
    """A tensor that says that it is on the GPU: what is refused is refused before anything follows its address."""
    is_cuda = property(lambda self: True)


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)


def ints(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnCard)


def books(**kw):
    d = dict(batch=4, max_blocks_per_seq=3, num_blocks=10, block_table=ints(4, 3), kv_len=ints(4), held=ints(4), shares=ints(10), free_ids=ints(10), free_count=ints(1))
    return dict(d, **kw)


WS = torch.zeros(16, dtype=torch.uint8)     # (too small for any of them)
CALLS = {
    "fork": lambda d: binding.ss_block_fork(d, ints(2), ints(2), None, ints(2), ints(2), ints(1), WS),
    "release": lambda d: binding.ss_block_release(d, ints(1), WS),
    "compact": lambda d: binding.ss_block_compact(d, None, ints(5), ints(5), ints(1), ints(1), WS),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("name,x,text", [
    ("kv_len", ints(4, dtype=torch.int64), "int64"), ("kv_len", ints(3), "at least 4"), ("kv_len", ints(8)[::2], "strides"), ("kv_len", torch.zeros(4, dtype=torch.int32), "on cpu"),
    ("held", ints(4, dtype=torch.int64), "int64"), ("held", ints(3), "at least 4"), ("shares", ints(10, dtype=torch.float32), "float32"), ("shares", ints(9), "at least 10"),
    ("block_table", ints(3, 4).T, "strides"), ("block_table", ints(11), "at least 12"), ("free_ids", ints(9), "at least 10"), ("free_ids", ints(10, dtype=torch.int64), "int64"),
    ("free_count", ints(1, dtype=torch.int64), "int64"), ("free_count", ints(0), "at least 1")])
def test_books_that_are_not_what_their_addresses_say(call, name, x, text):
    with pytest.raises(binding.SpecVerifyError, match=f"{name} must be .*{text}"):
        CALLS[call](books(**{name: x}))


@pytest.mark.parametrize("call", CALLS)
def test_books_that_are(call):
    with pytest.raises(binding.SpecVerifyError, match="workspace"):      # (the library's own refusal)
        CALLS[call](books())


def test_compaction_without_shares():
    with pytest.raises(binding.SpecVerifyError, match="workspace"):
        CALLS["compact"](books(shares=None))
    for call in ("fork", "release"):
        with pytest.raises((binding.SpecVerifyError, AttributeError)):
            CALLS[call](books(shares=None))
