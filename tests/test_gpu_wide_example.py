"""The end-to-end example with wide draft trees and shared prompts must run as shipped and keep its books."""
import numpy as np
import pytest

from paper_2604_09562_amd import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes,samples", [(48, 3), (70, 1), (1, 2)])
def test_example_wide_trees(nodes, samples):
    r = example.run_wide(steps=4, batch=3, layers=2, nodes=nodes, samples=samples, vocab=4096, seed=5, verbose=False)
    live = r["live"]
    assert live.sum() == (3 * (samples - 1) if samples > 1 else 3)
    assert np.all(r["emitted"] >= np.where(live, 4, 2))
    # every emitted token but the one still in flight has become a valid cache position
    assert np.array_equal((r["kv_len"] - r["start_len"])[live], r["emitted"][live]) and np.all(r["kv_len"][~live] == 0)
    assert r["used"] <= r["held"] and (samples < 3 or r["used"] < r["held"])
