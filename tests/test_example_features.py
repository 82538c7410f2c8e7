"""What the example's policy reads of a graph."""
import os
import sys

import numpy as np

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import learn_placement as example  # noqa: E402
from workloads import make_workload  # noqa: E402


def test_vertices_in_topological_order():
    w = make_workload("tiny")
    table, order = example.features(w)
    assert table.shape == (w.n, 6) and np.isfinite(table.numpy()).all()
    assert sorted(order.tolist()) == list(range(w.n))
    at = np.empty(w.n, dtype=np.int64)
    at[order.numpy()] = np.arange(w.n)
    tails = np.repeat(np.arange(w.n), np.diff(w.succ_ptr))
    assert (at[tails] < at[w.succ_idx]).all()


def test_policy_has_a_logit_per_device():
    p = example.Policy(5, width=16, blocks=3)
    assert p.head.shape == (16, 5) and len(p.into) == 3 and p.into[0].shape == (16, 48)
