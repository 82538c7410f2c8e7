"""The operators of a learned placement policy in 64 bits on the CPU, written from their formulas row by row, and how far a
kernel that works in 32 bits may be from them.

A tolerance is what rounding can cost: U = 2^-24 for each operation in 32 bits (with a small factor for the operations of
a formula, the error of the hardware's exp and reciprocal and the sums inside a workgroup), carried through the formula
by the absolute values of its terms, and half a step of the result's type at the end."""
import numpy as np
import torch

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype, ref):
    """The last rounding; values below the type's normal range are rounded to its smallest step."""
    fi = torch.finfo(dtype)
    ref = np.where(np.isfinite(ref), ref, 0.0)
    return fi.eps / 2 * np.abs(ref) + fi.tiny * fi.eps


def near(got, ref, tol, what=""):
    """Every element within its tolerance; infinities and NaN where the reference has them."""
    g, r = got.detach().cpu().double().numpy().reshape(-1), np.asarray(ref, dtype=np.float64).reshape(-1)
    t = np.broadcast_to(np.asarray(tol, dtype=np.float64), np.shape(ref)).reshape(-1)
    assert g.shape == r.shape, (what, g.shape, r.shape)
    r = np.where(np.abs(r) > torch.finfo(got.dtype).max, np.copysign(np.inf, r), r)      # what the type cannot hold
    odd = ~np.isfinite(r)
    assert np.array_equal(np.isnan(g), np.isnan(r)), what
    inf = np.isinf(r)
    assert np.array_equal(g[inf], r[inf]), what
    with np.errstate(invalid="ignore"):
        off = np.where(odd, -1, np.abs(g - r) - t)
    bad = np.nonzero(~(off <= 0))[0]
    assert bad.size == 0, f"{what}: {bad.size} of {g.size} off, first at {bad[0]}: {g[bad[0]]} for {r[bad[0]]} +- {t[bad[0]]}"


def wide(t):
    return None if t is None else t.detach().cpu().double().numpy()


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1, e) / (1 + e)


# ---- recurrence --------------------------------------------------------------------------------------


def recurrence(f, x, ptr, bias=None, h0=None, reverse=False, dh=None, dlast=None):
    """Row by row.  Returns values and tolerances (before the last rounding) by name."""
    f, x = wide(f), wide(x)
    N, D = f.shape
    S = len(ptr) - 1
    if bias is not None:
        f = f + wide(bias)
    h0 = np.zeros((S, D)) if h0 is None else wide(h0)
    a, z = sigmoid(f), sigmoid(-f)
    h, before, last = np.zeros((N, D)), np.zeros((N, D)), h0.copy()
    eh, eb, el = np.zeros((N, D)), np.zeros((N, D)), np.zeros((S, D))
    for s in range(S):
        rows = list(range(ptr[s], ptr[s + 1]))
        if reverse:
            rows.reverse()
        state, err = h0[s].copy(), np.zeros(D)
        most = np.maximum(np.abs(h0[s]), np.abs(x[rows]).max(0) if rows else 0)
        for t in rows:
            before[t], eb[t] = state, err
            # z off by a few U relative to itself (its exponent by U times itself), the step's products and sums off by U of
            # what they join; a run's product of a and its state from zero are no larger than what they stand for
            err = a[t] * err + U * most * (8 * z[t] * (2 + np.abs(f[t])) + 8)
            state = a[t] * state + z[t] * x[t]
            h[t], eh[t] = state, err
        last[s], el[s] = state, err
    out, tol = {"h": h, "last": last}, {"h": eh, "last": el}
    if dh is None:
        return out, tol
    dh = wide(dh)
    dlast = np.zeros((S, D)) if dlast is None else wide(dlast)
    g, eg, size = np.zeros((N, D)), np.zeros((N, D)), np.zeros((N, D))
    dh0, eu0 = dlast.copy(), np.zeros((S, D))
    for s in range(S):
        rows = list(range(ptr[s], ptr[s + 1]))
        if not reverse:
            rows.reverse()
        u, err, big = dlast[s].copy(), np.zeros(D), np.abs(dlast[s])
        for t in rows:
            g[t], size[t] = dh[t] + u, np.abs(dh[t]) + big
            eg[t] = err + U * size[t]
            u, big = a[t] * g[t], a[t] * size[t]
            err = a[t] * eg[t] + U * size[t] * (8 * z[t] * (2 + np.abs(f[t])) + 8)
        dh0[s], eu0[s] = u, err
    slack = 16 * U * (2 + np.abs(f))
    out["dx"], tol["dx"] = z * g, z * (eg + slack * size)
    out["df"] = g * (before - x) * a * z
    mag = np.abs(before) + np.abs(x)
    tol["df"] = a * z * (eg * mag + size * eb + slack * size * mag)
    out["dbias"] = out["df"].sum(0)
    tol["dbias"] = tol["df"].sum(0) + 32 * U * np.abs(out["df"]).sum(0)
    out["dh0"], tol["dh0"] = dh0, eu0
    return out, tol


# ---- norms, gate and residual ------------------------------------------------------------------------


def joint(x, y, gate, w_pre, w_post, act, scale, eps, dr=None, dz=None):
    x, y, gate, w_pre, w_post = (wide(v) for v in (x, y, gate, w_pre, w_post))
    many = 64 * U
    out, tol = {}, {}
    value = slope = np.ones(1)
    if gate is not None:
        sg = sigmoid(gate)
        value, slope = {"none": (gate, np.ones(1)), "sigmoid": (sg, sg * (1 - sg)),
                        "silu": (gate * sg, sg * (1 + gate * (1 - sg)))}[act]
        steep = 2 + np.abs(gate)            # an exponent's error
    else:
        steep = 2
    r = x.copy()
    off = U * np.abs(x)
    ry = yh = u = None
    if y is not None:
        u = y
        if w_post is not None:
            ry = 1 / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
            yh = y * ry
            u = yh * w_post
        r = x + scale * value * u
        off = off + many * steep * np.abs(scale * value * u)
    rr = 1 / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    rh = r * rr
    # an error of r moves z by itself and through the mean
    off_rh = rr * (off + np.abs(rh) * np.sqrt((off ** 2).mean(-1, keepdims=True))) + many * np.abs(rh)
    out["r"], tol["r"] = r, off + U * np.abs(r)
    out["z"], tol["z"] = rh * w_pre, np.abs(w_pre) * off_rh
    if dz is None:
        return out, tol
    dz = wide(dz)
    dr = np.zeros_like(x) if dr is None else wide(dr)
    wd = w_pre * dz
    dot, absdot = (wd * rh).mean(-1, keepdims=True), np.abs(wd * rh).mean(-1, keepdims=True)
    q = dr + rr * (wd - rh * dot)
    off_dot = (np.abs(wd) * off_rh).mean(-1, keepdims=True) + many * absdot
    size = np.abs(dr) + rr * (np.abs(wd) + np.abs(rh) * absdot)
    off_q = many * size + rr * (off_rh * np.abs(dot) + np.abs(rh) * off_dot) + rr * np.abs(wd) * many
    out["dx"], tol["dx"] = q, off_q
    out["dw_pre"] = (dz * rh).sum(0)
    tol["dw_pre"] = (np.abs(dz) * off_rh).sum(0) + 2 * many * np.abs(dz * rh).sum(0)
    if y is not None:
        du = q * scale * value
        off_du = np.abs(scale * value) * (off_q + many * steep * np.abs(q))
        if gate is not None:
            out["dgate"] = q * scale * u * slope
            steep_slope = np.abs(slope) + (np.abs(gate) + 1) * U if act == "none" else sg * (1 + np.abs(gate))
            tol["dgate"] = np.abs(scale * u) * (np.abs(slope) * off_q + many * steep * steep_slope * np.abs(q))
        if w_post is not None:
            out["dw_post"] = (du * yh).sum(0)
            tol["dw_post"] = (off_du * np.abs(yh)).sum(0) + 2 * many * np.abs(du * yh).sum(0)
            v, off_v = du * w_post, off_du * np.abs(w_post)
            dot2 = (v * yh).mean(-1, keepdims=True)
            off2 = (off_v * np.abs(yh)).mean(-1, keepdims=True) + many * np.abs(v * yh).mean(-1, keepdims=True)
            out["dy"] = ry * (v - yh * dot2)
            tol["dy"] = ry * (off_v + np.abs(yh) * off2 + many * (np.abs(v) + np.abs(yh * dot2)))
        else:
            out["dy"], tol["dy"] = du, off_du
    return out, tol


# ---- log probabilities of given tokens -----------------------------------------------------------------


def logprobs(logits, tokens, scale, allowed=None, top=0, dlogp=None, dentropy=None):
    x = wide(logits)
    R, V = x.shape
    allowed = np.ones((R, V), bool) if allowed is None else allowed
    x = np.where(allowed, x, -np.inf)
    tok = np.zeros((R, 0), np.int64) if tokens is None else tokens.cpu().numpy().astype(np.int64).reshape(R, -1)
    G = tok.shape[1]
    logp, tol_lp = np.zeros((R, G)), np.zeros((R, G))
    ent, tol_ent = np.zeros(R), np.zeros(R)
    top_idx, top_lp = np.full((R, top), -1), np.full((R, top), -np.inf)
    grad, tol_g = np.zeros((R, V)), np.zeros((R, V))
    dl = None if dlogp is None else wide(dlogp).reshape(R, G)
    de = np.zeros(R) if dentropy is None else wide(dentropy)
    with np.errstate(all="ignore"):
        for i in range(R):
            m = x[i].max() if not np.isnan(x[i]).any() else np.nan
            if m == -np.inf:
                logp[i] = np.where(tok[i] >= 0, -np.inf, 0.0)
                continue
            d = (x[i] - m) * scale
            e = np.exp(d)
            lp = d - np.log(e.sum())
            p = np.exp(lp)
            fin = np.isfinite(lp)
            ent[i] = -(p[fin] * lp[fin]).sum() if not np.isnan(m) and m != np.inf else np.nan
            # what e's exponents and a workgroup's sums cost
            tol_ent[i] = 400 * U * (1 + abs(ent[i]))
            one = U * (200 + 4 * np.abs(d))
            for g in range(G):
                if 0 <= tok[i, g] < V:
                    logp[i, g], tol_lp[i, g] = lp[tok[i, g]], one[tok[i, g]]
            order = np.argsort(-np.where(np.isnan(x[i]), np.inf, x[i]), kind="stable")[:top]
            for k, v in enumerate(order):
                if x[i, v] > -np.inf:
                    top_idx[i, k], top_lp[i, k] = v, lp[v]
            if dl is None:
                continue
            ok = (tok[i] >= 0) & (tok[i] < V)
            ok &= np.where(ok, x[i][np.where(ok, tok[i], 0)] > -np.inf, False)
            hits, ahits = np.zeros(V), np.zeros(V)
            np.add.at(hits, tok[i][ok], dl[i][ok])
            np.add.at(ahits, tok[i][ok], np.abs(dl[i][ok]))
            total, atotal = dl[i][ok].sum(), np.abs(dl[i][ok]).sum()
            safe = np.where(fin, lp, 0.0)
            if np.isnan(m) or m == np.inf:
                grad[i] = np.nan
                continue
            grad[i] = scale * (hits - p * total - de[i] * p * (safe + ent[i]))
            size = ahits + p * (atotal + abs(de[i]) * (np.abs(safe) + ent[i]))
            with np.errstate(invalid="ignore"):
                tol_g[i] = scale * (64 * U * size + np.where(fin, one, 0.0) * p * (atotal + abs(de[i]) * (1 + np.abs(safe) + ent[i])))
    out = {"logp": logp, "entropy": ent, "top_logp": top_lp, "top_idx": top_idx, "dlogits": grad}
    return out, {"logp": tol_lp, "entropy": tol_ent, "dlogits": tol_g}


def pack_mask(allowed):
    """bool [rows][vocab] as int64 words [rows][ceil(vocab/64)]."""
    R, V = allowed.shape
    bits = np.zeros((R, -(-V // 64) * 64), bool)
    bits[:, :V] = allowed
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int64).copy())
