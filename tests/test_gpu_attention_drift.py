"""States of cp_linear_attention over many steps, segments and chunks: decays close to one, whose rounding would add up, and decays of a state
alone.

Errors of rounding are as often above as below; what adds up is told by the part of a state's error that points along the state,
c = <S - ref, ref> / <ref, ref>.  Each rounding is off by at most U = 2^-24 of its value, so that the sum of n roundings of each of M normal values
has along the state a standard deviation of at most U sqrt(3 n / M), of which six are allowed (Hoeffding: 3e-8 to be further off)."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from attention_util import reference
from policy_util import TYPES, U, half_step, near, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SLOW = [-1e-5, -1e-6, -7e-6, -3e-5, -2e-4]


def along(got, ref):
    return abs(float(((wide(got) - ref) * ref).sum() / (ref * ref).sum()))


def allowed(roundings, values, log_decay, rows):
    # (gamma^n - 1 is off by at most 2^-21 of itself: expm1 and its argument)
    return 6 * U * np.sqrt(3 * roundings / values) + 2.0 ** -21 * abs(log_decay) * rows


def alike(log_decay, steps):
    """What the roundings of successive steps add where they are no longer independent of each other.  A step takes m |log_decay| of a state's
    last places from it, m from 2^23 to 2^24, and what is rounded off is the fraction of that.  Here m changes by 1/64 of itself a step (states of
    64, what is added of 1): the fraction moves by 2^23 |log_decay| / 64 and more, which makes it another one if that is above a half.  Below, at
    -1e-6 by 0.13, the same fraction is rounded off again and again, at most half a last place or U of the state each time, the same way.  (The
    formula with correct rounding, on the CPU, is off by 2.2e-6 there, and by at most 2.2e-7 for the other decays.)"""
    return steps * U if 2.0 ** 23 * abs(log_decay) / 64 < 0.5 else 0.0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_steps(dtype):
    N, H, K = 4000, len(SLOW), 64
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(N, H, K, generator=g).to(TYPES[dtype]) for _ in range(3))
    h0 = torch.randn(1, H, K, K, generator=g) * 64
    log_decay = torch.tensor(SLOW)
    gamma, ref = np.exp(wide(log_decay))[:, None, None], wide(h0)[0]
    for t in range(N):
        ref = gamma * ref + wide(k[t])[:, :, None] * wide(v[t])[:, None, :]
    q, k, v, state, log_decay = (t.to(DEV) for t in (q, k, v, h0, log_decay))
    last = cpe.cp_linear_attention(q, k, v, log_decay, h0=state, want_last=True)["last"]
    state = state.clone()
    for t in range(N):
        cpe.cp_linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], state, log_decay)
    for h in range(H):
        # a step rounds a state twice
        assert along(state[0, h], ref[h]) <= allowed(2 * N, K * K, SLOW[h], N) + alike(SLOW[h], N), ("step", SLOW[h], along(state[0, h], ref[h]))
        assert along(last[0, h], ref[h]) <= allowed(2 * N, K * K, SLOW[h], N), ("last", SLOW[h], along(last[0, h], ref[h]))


@pytest.mark.parametrize("low", [-1e-6, -3e-6, -1e-5])
def test_segments(low):
    # 1,024 segments of 128 rows of one head: two roundings each, and the last segment's chunks
    N, K = 131072, 64
    g = torch.Generator().manual_seed(2)
    q, k, v, do = (torch.randn(N, 1, K, generator=g) for _ in range(4))
    h0, dlast = (torch.randn(1, 1, K, K, generator=g) * 4096 for _ in range(2))
    log_decay = torch.tensor([low])
    worn = np.exp(float(log_decay[0]) * np.arange(N + 1))
    last = worn[N] * wide(h0)[0, 0] + (wide(k)[:, 0] * worn[N - 1::-1, None]).T @ wide(v)[:, 0]
    dh0 = worn[N] * wide(dlast)[0, 0] + (wide(q)[:, 0] * worn[1:, None]).T @ wide(do)[:, 0]
    q, k, v, do, h0, dlast, log_decay = (t.to(DEV) for t in (q, k, v, do, h0, dlast, log_decay))
    out = cpe.cp_linear_attention(q, k, v, log_decay, h0=h0, want_last=True, want_carry=True)
    assert out["carry"].shape[0] == 1024
    back = cpe.cp_linear_attention_backward(do, q, k, v, log_decay, out["carry"], h0=h0, dlast=dlast)
    for got, ref, name in ((out["last"], last, "last"), (back["dh0"], dh0, "dh0")):
        assert along(got[0, 0], ref) <= allowed(2 * 1030, K * K, low, N), (name, along(got[0, 0], ref))


@pytest.mark.parametrize("N", [1, 5, 33, 64, 70, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_state_that_nothing_is_added_to(dtype, N):
    # each chunk multiplies it by a power of gamma that is off by at most 2^-22, and rounds
    log_decay = torch.tensor([-0.3, -0.69, -0.7, -2.0, -5.0])
    H, K, V = 5, 32, 40
    g = torch.Generator().manual_seed(N)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k, v, do = r(N, H, K), torch.zeros(N, H, K), r(N, H, V), torch.zeros(N, H, V)
    q, k, v, do = (t.to(TYPES[dtype]).to(DEV) for t in (q, k, v, do))
    h0, dlast = r(1, H, K, V), r(1, H, K, V)
    kw = dict(h0=h0.to(DEV))
    out = cpe.cp_linear_attention(q, k, v, log_decay.to(DEV), want_last=True, want_carry=True, **kw)
    back = cpe.cp_linear_attention_backward(do, q, k, v, log_decay.to(DEV), out["carry"], dlast=dlast.to(DEV), **kw)
    state = h0.to(DEV)
    for t in range(N):
        cpe.cp_linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], state, log_decay.to(DEV))
    gamma = np.exp(wide(log_decay) * N)[None, :, None, None]
    for got, ref, times, name in ((out["last"], gamma * wide(h0), N // 32 + 2, "last"), (back["dh0"], gamma * wide(dlast), N // 32 + 2, "dh0"),
                                  (state, gamma * wide(h0), N, "state")):
        # (what is below the least normal number may be 0)
        off = np.abs(wide(got) - ref) - (times * 2.0 ** -21 * np.abs(ref) + 2.0 ** -126)
        assert (off <= 0).all(), (name, float((np.abs(wide(got) - ref) / np.abs(ref)).max()))


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("first", [40, 64, 100, 190])
@pytest.mark.parametrize("dtype", TYPES)
def test_decays_gradient_of_a_state_that_nothing_is_added_to(dtype, first, reverse):
    # what the outputs from row `first` on read has come through the rows before, each of which counts once more for the decays' gradient
    N, H, K, V = 200, 6, 24, 40
    g = torch.Generator().manual_seed(first)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k, v, do = r(N, H, K), torch.zeros(N, H, K), r(N, H, V), r(N, H, V)
    do[slice(N - first, N) if reverse else slice(0, first)] = 0
    q, k, v, do = (t.to(TYPES[dtype]).to(DEV) for t in (q, k, v, do))
    log_decay, h0 = torch.tensor([-0.01, -0.2, -0.3, -0.44, -0.6, -0.8], device=DEV), r(1, H, K, V).to(DEV)
    kw = dict(h0=h0, reverse=reverse)
    carry = cpe.cp_linear_attention(q, k, v, log_decay, want_carry=True, **kw)["carry"]
    got = cpe.cp_linear_attention_backward(do, q, k, v, log_decay, carry, **kw)
    ref, tol = reference(q, k, v, log_decay, [0, N], 1.0, h0, reverse, do)
    # (what is below the least normal number may be 0)
    near(got["dlog_decay"], ref["dlog_decay"], tol["dlog_decay"] + half_step(torch.float32, ref["dlog_decay"]) + N * N * K * V * 2.0 ** -126, "dlog_decay")
