"""Linear attention in 64 bits on the CPU, row by row, with its gradient, and how far a kernel that works in 32 bits may be from it.

Tolerances follow the formula's terms by their absolute values (the same recurrences over |q|, |k|, |v|).  What each costs:
sums and decays in 32 bits U = 2^-24 for each of a row's products, a chunk's rows and the chunks that a state has passed; for
16-bit types, whose products are exact, the states and scores that go into products as two bf16: each is off by half a step of the
second, 2^-16 of it, a state by as much again from the rows it was made of, and for fp16 (two bf16 itself) the product of both
second parts, at most 2^-16, is left out of each: 2^-14 in all."""
import numpy as np
import torch

from policy_util import U, wide


def split_cost(dtype):
    return 0.0 if dtype == torch.float32 else 2.0 ** -14


def reference(q, k, v, log_decay, ptr, scale=1.0, h0=None, reverse=False, do=None, dlast=None):
    """Values and tolerances (before the last rounding) by name."""
    dtype = q.dtype
    q, k, v = wide(q), wide(k), wide(v)
    N, H, K = q.shape
    KV, V = v.shape[1:]
    G, S = H // KV, len(ptr) - 1
    gamma = np.ones(H) if log_decay is None else np.exp(wide(log_decay))
    k, v = np.repeat(k, G, 1), np.repeat(v, G, 1)
    h0 = np.zeros((S, H, K, V)) if h0 is None else wide(h0)
    g3 = gamma[:, None, None]
    lost = split_cost(dtype)
    out = {"o": np.zeros((N, H, V)), "last": h0.copy()}
    size = {"o": np.zeros((N, H, V)), "last": np.abs(h0)}
    steps = np.zeros(N)                          # rows that a row's state has come through
    grad = do is not None
    if grad:
        do = wide(do)
        dlast = np.zeros((S, H, K, V)) if dlast is None else wide(dlast)
        for name, shape in (("dq", (N, H, K)), ("dk", (N, H, K)), ("dv", (N, H, V)), ("dlog_decay", (H,))):
            out[name], size[name] = np.zeros(shape), np.zeros(shape)
        out["dh0"], size["dh0"] = dlast.copy(), np.abs(dlast)
    order = []
    with np.errstate(invalid="ignore", over="ignore"):
        for s in range(S):
            rows = list(range(ptr[s], ptr[s + 1]))
            if reverse:
                rows.reverse()
            order.append(rows)
            state, big = h0[s].copy(), np.abs(h0[s])
            kept = []
            for n, t in enumerate(rows):
                kept.append((g3 * state, g3 * big))
                add = k[t][:, :, None] * v[t][:, None, :]
                state, big = g3 * state + add, g3 * big + np.abs(add)
                out["o"][t] = scale * np.einsum("hk,hkv->hv", q[t], state)
                size["o"][t] = abs(scale) * np.einsum("hk,hkv->hv", np.abs(q[t]), big)
                steps[t] = n
                if grad:
                    out["dq"][t] = scale * np.einsum("hv,hkv->hk", do[t], state)
                    size["dq"][t] = abs(scale) * np.einsum("hv,hkv->hk", np.abs(do[t]), big)
            out["last"][s], size["last"][s] = state, big
            if not grad:
                continue
            d, big = dlast[s].copy(), np.abs(dlast[s])
            for t, (before, before_big) in zip(rows[::-1], kept[::-1]):
                add = scale * q[t][:, :, None] * do[t][:, None, :]
                d, big = d + add, big + np.abs(add)
                out["dv"][t], size["dv"][t] = np.einsum("hk,hkv->hv", k[t], d), np.einsum("hk,hkv->hv", np.abs(k[t]), big)
                out["dk"][t], size["dk"][t] = np.einsum("hv,hkv->hk", v[t], d), np.einsum("hv,hkv->hk", np.abs(v[t]), big)
                out["dlog_decay"] += (d * before).sum((1, 2))
                size["dlog_decay"] += (big * before_big).sum((1, 2))
                d, big = g3 * d, g3 * big
            out["dh0"][s], size["dh0"][s] = d, big
    longest = max([len(r) for r in order] + [0])
    cost = lost + U * (K + V + 128 + longest / 8)
    tol = {n: a * cost for n, a in size.items()}
    if grad:
        # (rows' terms are weighted by how far apart they are, once more a product, and summed in 64 bits)
        tol["dlog_decay"] *= 2
        for n in ("dk", "dv"):
            out[n], tol[n] = out[n].reshape(N, KV, G, -1).sum(2), tol[n].reshape(N, KV, G, -1).sum(2) + G * U * np.abs(out[n]).reshape(N, KV, G, -1).sum(2)
    return out, tol
