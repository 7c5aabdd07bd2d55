"""What ties a counter summary to the streaming kernel is the sources that it is built from: declarations of the cache's writes, which it never reads, stand elsewhere."""
import os

import bench

from .helpers import CSRC


def test_hashed_sources_hold_nothing_of_the_cache_writes():
    assert len(bench.attn_source_hash()) == 16
    for name in bench.ATTN_SOURCES:
        text = open(os.path.join(CSRC, name)).read()
        for other in ("KvAppendArgs", "kv_append_launch", "kv_compact_launch", "kv_commit_launch"):
            assert other not in text, (name, other)
