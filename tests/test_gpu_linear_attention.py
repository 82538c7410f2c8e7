"""cp_linear_attention, its gradient and its step against the recurrence in 64 bits, row by row."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from attention_util import reference, split_cost
from policy_util import TYPES, U, half_step, near, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(N, H, KV, K, V, dtype, S=1, seed=0, h0=False, grad=False, fast=0.7, slow=2e-4):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    dt = TYPES[dtype]
    i = dict(q=r(N, H, K).to(dt), k=r(N, KV, K).to(dt), v=r(N, KV, V).to(dt),
             log_decay=-torch.exp(torch.empty(H).uniform_(np.log(slow), np.log(fast), generator=g)))
    i["h0"] = r(S, H, K, V) if h0 else None
    if grad:
        i["do"], i["dlast"] = r(N, H, V).to(dt), r(S, H, K, V) if h0 else None
    return {n: t.to(DEV) if t is not None else None for n, t in i.items()}


def rounded(name, ref, tol, dtype):
    wide_out = name in ("last", "dlog_decay", "dh0")
    return tol[name] + half_step(torch.float32 if wide_out else dtype, ref[name])


def check(i, ptr, scale=0.25, reverse=False, seq_ptr=None, batch=None, out=None):
    kw = dict(scale=scale, seq_ptr=seq_ptr, h0=i["h0"], reverse=reverse)
    lead = (lambda t: t.view(batch, -1, *t.shape[1:])) if batch else (lambda t: t)
    grad = "do" in i
    got = cpe.cp_linear_attention(lead(i["q"]), lead(i["k"]), lead(i["v"]), i["log_decay"], want_last=True, want_carry=grad, **kw)
    ref, tol = reference(i["q"], i["k"], i["v"], i["log_decay"], ptr, scale, i["h0"], reverse, i.get("do"), i.get("dlast"))
    if grad:
        got.update(cpe.cp_linear_attention_backward(lead(i["do"]), lead(i["q"]), lead(i["k"]), lead(i["v"]), i["log_decay"], got["carry"],
                                                    dlast=i["dlast"], **kw))
    for name in ref:
        if name in got:
            near(got[name], ref[name], rounded(name, ref, tol, i["q"].dtype), name)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 63, 64, 65, 127, 200, 331])
def test_lengths(N, dtype):
    check(make(N, 2, 2, 32, 32, dtype, seed=N, h0=N % 2 == 0, grad=True), [0, N])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,V", [(1, 1), (3, 5), (16, 100), (33, 64), (64, 65), (65, 128), (128, 128), (129, 40), (200, 130), (256, 256), (31, 255)])
def test_widths(K, V, dtype):
    check(make(150, 2, 1, K, V, dtype, seed=K, h0=True, grad=True), [0, 150])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("H,KV", [(1, 1), (4, 4), (6, 2), (5, 1)])
def test_packed_sequences(H, KV, reverse):
    cuts = [0, 0, 1, 1, 3, 70, 70, 134, 262, 400, 400, 777, 778, 778]
    i = make(778, H, KV, 24, 40, "fp32", S=len(cuts) - 1, seed=H, h0=True, grad=True)
    check(i, cuts, reverse=reverse, seq_ptr=torch.tensor(cuts, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_packed_sequences_in_16_bits(dtype):
    cuts = [0, 5, 200, 200, 611]
    i = make(611, 3, 3, 64, 96, dtype, S=4, seed=5, h0=True, grad=True)
    check(i, cuts, seq_ptr=torch.tensor(cuts, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("batch,N", [(1, 1300), (3, 1000), (5, 129), (7, 1)])
def test_equal_sequences(batch, N, reverse):
    i = make(batch * N, 2, 2, 40, 72, "bf16", S=batch, seed=N, h0=True, grad=True)
    check(i, [s * N for s in range(batch + 1)], reverse=reverse, batch=batch)


@pytest.mark.parametrize("dtype", TYPES)
def test_steps(dtype):
    g = torch.Generator().manual_seed(3)
    for S, H, KV, K, V in ((1, 1, 1, 1, 1), (3, 4, 2, 33, 65), (9, 3, 1, 128, 128), (5, 2, 2, 256, 256), (4, 2, 2, 16, 255)):
        i = make(S, H, KV, K, V, dtype, seed=K)
        pool = S + 3
        state = torch.randn(pool, H, K, V, generator=g).to(DEV)
        slots = torch.randperm(pool, generator=g)[:S].to(torch.int32)
        if S > 2:
            slots[1] = -1
        before = wide(state)
        got = cpe.cp_linear_attention_step(i["q"], i["k"], i["v"], state, i["log_decay"], scale=0.5, slots=slots.to(DEV))
        after, o, size = before.copy(), np.zeros((S, H, V)), np.zeros((S, H, V))
        gamma = np.exp(wide(i["log_decay"]))[:, None, None]
        q, k, v = wide(i["q"]), np.repeat(wide(i["k"]), H // KV, 1), np.repeat(wide(i["v"]), H // KV, 1)
        for n, slot in enumerate(slots.tolist()):
            if slot >= 0:
                add = k[n][:, :, None] * v[n][:, None, :]
                after[slot] = gamma * before[slot] + add
                big = np.abs(gamma * before[slot]) + np.abs(add)
                o[n] = 0.5 * np.einsum("hk,hkv->hv", q[n], after[slot])
                size[n] = 0.5 * np.einsum("hk,hkv->hv", np.abs(q[n]), big)
        near(got["o"], o, size * U * (K + 8) + half_step(i["q"].dtype, o), "o")
        near(state, after, 8 * U * (np.abs(before) + np.abs(after)), "state")
