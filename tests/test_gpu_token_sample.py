"""cp_token_sample against its definition in 64 bits, row by row."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from policy_util import TYPES, U, pack_mask, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def kept_places(x, allowed, scale, top_k, top_p, min_p):
    """(probabilities of the kept places in units of the best one's, by place; None where nothing can be drawn)"""
    x = np.where(allowed, x, -np.inf)
    if not allowed.any() or np.isnan(x).any() or x.max() in (np.inf, -np.inf):
        return None
    p = np.exp((x - x.max()) * scale)
    order = np.argsort(-x, kind="stable")
    if top_k:
        order = order[:top_k]
    total, ahead, kept = p[order].sum(), 0.0, []
    for v in order:
        if top_p < 1 and kept and not ahead < top_p * total:
            break
        kept.append(v)
        ahead += p[v]
    out = np.zeros_like(p)
    out[kept] = np.where(p[kept] >= min_p, p[kept], 0.0)
    return out


def check(logits, u, allowed=None, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, dtype=torch.int64, **kw):
    R, V = logits.shape
    each = lambda v, t: torch.tensor(v, dtype=t, device=DEV) if isinstance(v, (list, np.ndarray)) else v  # noqa: E731
    got = cpe.cp_token_sample(logits.to(DEV), u.to(DEV), allow=None if allowed is None else pack_mask(allowed).to(DEV), scale=each(scale, torch.float32),
                              top_k=each(top_k, torch.int32), top_p=each(top_p, torch.float32), min_p=each(min_p, torch.float32), dtype=dtype,
                              want_logp=True, **kw)
    x, r = wide(logits), np.clip(np.nan_to_num(u.numpy(), nan=0.0), 0, np.float32(1 - 2.0 ** -24)).reshape(R, -1).astype(np.float64)
    at = lambda v, i: float(np.float32(v[i])) if isinstance(v, (list, np.ndarray)) else v  # noqa: E731
    tokens, logp = got["tokens"].cpu().numpy().reshape(R, -1), got["logp"].cpu().numpy().reshape(R, -1)
    for i in range(R):
        p = kept_places(x[i], np.ones(V, bool) if allowed is None else allowed[i], at(scale, i), int(at(top_k, i)), at(top_p, i), at(min_p, i))
        if p is None:
            assert (tokens[i] == (255 if dtype == torch.uint8 else -1)).all() and (logp[i] == 0).all(), i
            continue
        upto = p.cumsum()
        for g in range(r.shape[1]):
            v = int(np.searchsorted(upto, r[i, g] * upto[-1], side="right"))
            assert tokens[i, g] == v, (i, g, tokens[i, g], v)
            ref = np.log(p[v] / upto[-1])
            assert abs(logp[i, g] - ref) <= U * (abs(ref) + 2.0 ** -20), (i, g, logp[i, g], ref)
    return got


def inputs(R, V, G, dtype, seed=0, by=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, V, generator=g) * by).to(TYPES[dtype]), torch.rand(R, G, generator=g)


FILTERS = [dict(), dict(top_k=5), dict(top_p=0.8), dict(min_p=0.1), dict(top_k=17, top_p=0.6), dict(top_k=3, min_p=0.3), dict(top_p=0.95, min_p=0.02),
           dict(top_k=40, top_p=0.9, min_p=0.01), dict(top_k=1), dict(top_p=0.0), dict(min_p=1.0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130, 255, 256, 257, 1000, 5000])
def test_places(V, dtype):
    for n, f in enumerate(FILTERS):
        check(*inputs(9, V, 5, dtype, seed=V + n), scale=0.8, **f)


@pytest.mark.parametrize("V", [6, 50, 200, 700])
@pytest.mark.parametrize("G", [0, 1, 3, 64, 257])
def test_given(V, G):
    logits, u = inputs(5, V, max(G, 1), "fp32", seed=G)
    check(logits, u[:, :G], top_p=0.9)


@pytest.mark.parametrize("V", [3, 40, 256, 3001])
def test_equal_logits(V):
    # ties are broken by place, and sums of equal shares are whole numbers: borders are met exactly
    _, u = inputs(4, V, 40, "bf16", seed=V)
    u[:, :4] = torch.tensor([0.0, 0.25, 0.5, 0.75])
    logits = torch.zeros(4, V)
    logits[1] = -0.0
    logits[1, ::2] = 0.0
    logits[2] = torch.arange(V) % 3
    logits[3] = torch.finfo(torch.bfloat16).min
    for f in FILTERS + [dict(top_k=V // 2 + 1), dict(top_p=0.5), dict(top_k=8, top_p=0.25)]:
        check(logits.to(torch.bfloat16), u, **f)


@pytest.mark.parametrize("V", [10, 100, 400])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_and_odd_rows(V, dtype):
    g = np.random.default_rng(V)
    logits, u = inputs(12, V, 6, dtype, seed=V)
    allowed = g.random((12, V)) < 0.5
    allowed[0] = False
    allowed[1], allowed[1, V // 2] = False, True
    logits[2] = -float("inf")
    logits[3, allowed[3].argmax()] = float("nan")
    logits[4, allowed[4].argmax()] = float("inf")
    logits[5, ~allowed[5]] = float("nan")                # what lies at a place that is not allowed is not looked at
    logits[6, ~allowed[6]] = float("inf")
    logits[7, ::2] = -float("inf")
    logits[8] = torch.finfo(logits.dtype).min
    u[9] = torch.tensor([0.0, 1.0, 2.0, -1.0, float("nan"), 1 - 2.0 ** -24])
    for f in FILTERS:
        check(logits, u, allowed, **f)


@pytest.mark.parametrize("V", [12, 90, 900])
def test_settings_a_row(V):
    R = 16
    logits, u = inputs(R, V, 3, "fp16", seed=V)
    g = np.random.default_rng(V)
    kw = dict(scale=g.uniform(0.3, 2, R), top_k=g.integers(0, V + 5, R), top_p=np.where(g.random(R) < 0.3, 1.0, g.random(R)), min_p=g.random(R) * 0.2)
    check(logits, u, **kw)
    for name in kw:
        check(logits, u, **{name: kw[name]})


@pytest.mark.parametrize("V", [20, 300])
def test_settings_out_of_range(V):
    logits, u = inputs(8, V, 2, "fp32")
    f = lambda *v: torch.tensor(v, device=DEV)  # noqa: E731
    bad = dict(scale=f(1.0, 0.0, -1.0, float("nan"), float("inf"), 1.0, 1.0, 1.0), top_p=f(1.0, 1.0, 1.0, 1.0, 1.0, 1.5, 1.0, 1.0),
               min_p=f(0.0, 0.0, 0.0, 0.0, 0.0, 0.0, float("nan"), 0.0), top_k=torch.tensor([0, 0, 0, 0, 0, 0, 0, -3], dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        cpe.cp_token_sample(logits.to(DEV), u.to(DEV), **bad)
    got = cpe.cp_token_sample(logits.to(DEV), u.to(DEV), check_status=False, **bad)
    assert int(got["status"]) == 256
    assert (got["tokens"][1:] == -1).all()
    assert torch.equal(got["tokens"][0], cpe.cp_token_sample(logits.to(DEV), u.to(DEV))["tokens"][0])
    again = cpe.cp_token_sample(logits.to(DEV), u.to(DEV), scale=torch.ones(8, device=DEV), out=dict(status=got["status"]))
    assert int(again["status"]) == 0


@pytest.mark.parametrize("V", [8, 100, 600])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.int32, torch.int64])
def test_strides(V, dtype):
    if V > 255 and dtype == torch.uint8:
        pytest.skip("no room for the places")
    logits, u = inputs(33, V + 3, 14, "bf16", seed=V)
    want = cpe.cp_token_sample(logits[:, 1:-2].contiguous().to(DEV), u.to(DEV), top_p=0.9, dtype=dtype)["tokens"]
    rows = torch.full((14, 33), 77, dtype=dtype, device=DEV)
    wider = torch.full((33, 30), 77, dtype=dtype, device=DEV)
    big = logits.to(DEV)[:, 1:-2]
    ut = u.t().contiguous().to(DEV).t()
    cpe.cp_token_sample(big, ut, top_p=0.9, out=dict(tokens=rows.t()))
    cpe.cp_token_sample(big, ut, top_p=0.9, out=dict(tokens=wider[:, 1:29:2]))
    assert torch.equal(rows.t(), want) and torch.equal(wider[:, 1:29:2], want)
    wider[:, 1:29:2] = 77
    assert (wider == 77).all()
    same = cpe.cp_token_sample(big, ut[:, :1].expand(33, 14), top_p=0.9, dtype=dtype)["tokens"]
    assert torch.equal(same, want[:, :1].expand(33, 14))
    assert torch.equal(cpe.cp_token_sample(big, ut[:, 3], top_p=0.9, dtype=dtype)["tokens"], want[:, 3])
