"""cp_token_sample where top_p ends among very many unlikely places, whose masses are small and come to much: what is kept is told by the
last places that can be drawn.

The best place's mass is 1 and exact, those of all others are off by at most 2e-12 of themselves (rows of 2^26 places; less in shorter ones), and
the reference's sums, which take equal places together, by 2^-63 for each value that occurs: no border below lies as near as twice that to
the mass that is asked for."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from policy_util import TYPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U_NUMBERS = torch.tensor([[0.0, 0.25, 0.5, 0.9, 0.99, 0.999, 0.9999, 1 - 2.0 ** -20, 1 - 2.0 ** -24]])


class Row:
    """A row's places from the best on, equal ones by rising place, and what it draws."""

    def __init__(self, x):
        self.values, self.which, self.counts = np.unique(-x.double().numpy(), return_inverse=True, return_counts=True)
        self.order = np.argsort(self.which, kind="stable")
        self.x = x.view(1, -1).to(DEV)

    def check(self, top_p, scale=1.0, top_k=0):
        got = cpe.cp_token_sample(self.x, U_NUMBERS.to(DEV), top_p=top_p, scale=scale, top_k=top_k)["tokens"].cpu()
        p = np.exp((self.values[0] - self.values).astype(np.longdouble) * np.longdouble(scale))
        front = np.concatenate([[0], self.counts.cumsum()])
        start = np.concatenate([[np.longdouble(0)], (self.counts * p).cumsum()])
        order = self.order[:top_k] if top_k else self.order
        group = self.which[order]
        ahead = start[group] + (np.arange(len(order)) - front[group]) * p[group]
        total = ahead[-1] + p[group[-1]]
        want = np.longdouble(top_p) * total
        n = int(np.searchsorted(ahead, want))                            # the first that is not below
        near = float(np.abs(ahead[max(n - 1, 0):n + 2] - want).min() / total)
        assert near > 2 * (2e-12 * float(total - self.counts[0]) / float(total) + len(p) * 2.0 ** -63), near
        kept = np.zeros(len(self.which), np.longdouble)
        kept[order[:max(n, 1)]] = p[group[:max(n, 1)]]
        upto = kept.cumsum()
        assert got[0].tolist() == [int(np.searchsorted(upto, np.longdouble(float(u)) * upto[-1], side="right")) for u in U_NUMBERS[0]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [9001, 131072, (1 << 22) + 5])
def test_one_high_place_before_a_flat_tail(V, dtype):
    x = torch.full((V,), -17.25, dtype=TYPES[dtype])
    x[V // 3] = 0.0
    row = Row(x)
    for top_p in (1 - 1e-3, 1 - 2e-4, 0.95, 0.9, 0.885):
        row.check(top_p)
        row.check(top_p, top_k=V - 5)
        row.check(top_p, scale=0.7)


@pytest.mark.parametrize("dtype", TYPES)
def test_tails_of_many_values(dtype):
    V = 1 << 21
    g = torch.Generator().manual_seed(3)
    for lo, hi in ((-17.0, -11.0), (-40.0, -9.0), (-14.5, -14.0)):
        x = (torch.rand(V, generator=g) * (hi - lo) + lo).to(TYPES[dtype])
        x[[7, 70007, V - 1]] = torch.tensor([0.0, -1.0, 0.0], dtype=TYPES[dtype])
        row = Row(x)
        for top_p in (0.99, 0.999, 1 - 1e-5, 0.86):
            row.check(top_p)
            row.check(top_p, top_k=V // 2)


def test_the_widest_row():
    # 2^26 places: the best one alone would be kept if those of 2^-37 counted for nothing or for one unit of 2^-35
    V = 1 << 26
    x = torch.full((V,), -24.875, dtype=torch.bfloat16)
    x[12345] = 0.0
    row = Row(x)
    for top_p in (0.9985, 0.9995, 0.99999):
        row.check(top_p)
    row.check(0.9995, top_k=V - 100)
