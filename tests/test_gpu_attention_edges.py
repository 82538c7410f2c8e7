"""cp_linear_attention at the borders: strides, values that are no numbers, decays from none to all, rows behind the last sequence, long
sequences, offsets beyond 32 bits, graphs and streams; its differentiable form; and the operators of a policy run together."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from attention_util import reference
from paper_1711_01912_amd import autograd
from policy_util import TYPES, half_step, near, wide
from test_gpu_linear_attention import check, make, rounded
from workloads import make_workload

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import learn_placement as example  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GRADS = ("dq", "dk", "dv", "dlog_decay", "dh0")


def both(i, **kw):
    """All results of a call and of its gradient."""
    kw = dict(scale=0.25, h0=i["h0"], **kw)
    out = cpe.cp_linear_attention(i["q"], i["k"], i["v"], i["log_decay"], want_last=True, want_carry=True, **kw)
    out.update(cpe.cp_linear_attention_backward(i["do"], i["q"], i["k"], i["v"], i["log_decay"], out["carry"], dlast=i["dlast"], **kw))
    return {n: t for n, t in out.items() if n in ("o", "last") + GRADS}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,V", [(32, 32), (40, 72), (33, 7), (128, 128)])
def test_strides(K, V, dtype):
    N, H = 150, 3
    i = make(N, H, H, K, V, dtype, seed=K, h0=True, grad=True)
    want = both(i)
    W = 2 * K + V
    # slices of [rows][heads][q k v], of [rows][q k v] at an odd place, heads in front of rows
    inter, fused = torch.zeros(N, H, W + 3, dtype=i["q"].dtype, device=DEV), torch.zeros(N, H * W + 5, dtype=i["q"].dtype, device=DEV)
    for views in ([inter[..., :K], inter[..., K:2 * K], inter[..., 2 * K:W]],
                  [fused[:, 1:1 + H * K].unflatten(1, (H, K)), fused[:, 1 + H * K:1 + 2 * H * K].unflatten(1, (H, K)), fused[:, 1 + 2 * H * K:1 + H * W].unflatten(1, (H, V))],
                  [torch.zeros(H, N, w, dtype=i["q"].dtype, device=DEV).transpose(0, 1) for w in (K, K, V)]):
        for view, name in zip(views, "qkv"):
            view.copy_(i[name])
        got = both(dict(i, **dict(zip("qkv", views))))
        assert all(torch.equal(got[n], want[n]) for n in want)
        # and results there
        kw = dict(scale=0.25, h0=i["h0"])
        carry = cpe.cp_linear_attention(*views, i["log_decay"], want_carry=True, **kw)["carry"]
        to = [torch.zeros_like(v).as_strided(v.shape, v.stride()) if v.is_contiguous() else torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=DEV) for v in views]
        got = cpe.cp_linear_attention_backward(i["do"], *views, i["log_decay"], carry, dlast=i["dlast"], out=dict(zip(("dq", "dk", "dv"), to)), **kw)
        assert all(torch.equal(got[n], want[n]) for n in GRADS)
        o = torch.empty(H, N, V, dtype=i["q"].dtype, device=DEV).transpose(0, 1)
        assert torch.equal(cpe.cp_linear_attention(*views, i["log_decay"], out={"o": o}, **kw)["o"], want["o"])


def test_one_head_or_row_for_all():
    i = make(90, 4, 1, 24, 40, "fp32", seed=1, h0=True, grad=True)
    want = both(i)
    spread = dict(i, k=i["k"].expand(90, 4, 24), v=i["v"].expand(90, 4, 40))
    got = both(spread)
    assert torch.equal(got["o"], want["o"]) and torch.equal(got["last"], want["last"]) and got["dk"].shape == (90, 4, 24)
    ref, tol = reference(i["q"], i["k"], i["v"], i["log_decay"], [0, 90], 0.25, i["h0"], False, i["do"], i["dlast"])
    for n in ("dk", "dv"):
        near(got[n].double().sum(1, keepdim=True).float(), ref[n], tol[n] + half_step(torch.float32, ref[n]) + 4 * 2.0 ** -24 * wide(got[n].abs()).sum(1, keepdims=True), n)
    q = i["q"][:1].expand(90, 4, 24)
    assert torch.equal(cpe.cp_linear_attention(q, i["k"], i["v"], i["log_decay"])["o"], cpe.cp_linear_attention(q.contiguous(), i["k"], i["v"], i["log_decay"])["o"])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_behind_the_last_sequence(dtype, reverse):
    cuts = [0, 3, 140, 140, 300]
    i = make(777, 2, 1, 32, 48, dtype, S=4, seed=3, h0=True, grad=True)
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    for n in ("q", "k", "v", "do"):
        i[n][300:] = float("nan")
    kw = dict(scale=0.25, seq_ptr=ptr, h0=i["h0"], reverse=reverse)
    keep = {n: torch.full_like(t, 7.0) for n, t in (("o", i["do"]), ("dq", i["q"]), ("dk", i["k"]), ("dv", i["v"]))}
    fwd = cpe.cp_linear_attention(i["q"], i["k"], i["v"], i["log_decay"], want_last=True, want_carry=True, out={"o": keep["o"]}, **kw)
    bwd = cpe.cp_linear_attention_backward(i["do"], i["q"], i["k"], i["v"], i["log_decay"], fwd["carry"], dlast=i["dlast"],
                                           out={n: keep[n] for n in ("dq", "dk", "dv")}, **kw)
    for t in keep.values():
        assert (t[300:] == 7).all()
    cut = {n: t[:300] if n in ("q", "k", "v", "do") else t for n, t in i.items()}
    ref, tol = reference(cut["q"], cut["k"], cut["v"], i["log_decay"], cuts, 0.25, i["h0"], reverse, cut["do"], i["dlast"])
    for n, t in {**fwd, **bwd}.items():
        if n in ref:
            near(t[:300] if n in keep else t, ref[n], rounded(n, ref, tol, i["q"].dtype), n)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,K,V", [("fp32", 32, 32), ("bf16", 64, 128), ("fp16", 40, 48), ("bf16", 256, 64)])
def test_values_that_are_no_numbers(dtype, K, V, bad):
    N, H, at = 300, 3, 133
    cuts = [0, 250, 300]
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    i = make(N, H, H, K, V, dtype, S=2, seed=5, h0=True, grad=True)
    clean = both(i, seq_ptr=ptr)
    ref, tol = reference(i["q"], i["k"], i["v"], i["log_decay"], cuts, 0.25, i["h0"], False, i["do"], i["dlast"])
    for name in ("q", "k", "v", "do"):
        j = dict(i, **{name: i[name].clone()})
        j[name][at, 1, 2] = bad
        got = both(j, seq_ptr=ptr)
        # what the row's value does not flow into: o before it, and the gradients that look the other way; other heads and sequences
        before, after = slice(0, at), slice(at + 1, 250)
        reach = {"q": dict(o=slice(at, at + 1), dk=slice(0, at + 1), dv=slice(0, at + 1), dq=slice(0, 0)),
                 "k": dict(o=slice(at, 250), dq=slice(at, 250), dv=slice(at, at + 1), dk=slice(0, 0)),
                 "v": dict(o=slice(at, 250), dq=slice(at, 250), dk=slice(at, at + 1), dv=slice(0, 0)),
                 "do": dict(dq=slice(at, at + 1), dk=slice(0, at + 1), dv=slice(0, at + 1), o=slice(0, 0))}[name]
        for n in ("o", "dq", "dk", "dv"):
            others = [h for h in range(H) if h != 1]
            assert torch.equal(got[n][:, others], clean[n][:, others]), (name, n)
            assert torch.equal(got[n][250:], clean[n][250:]), (name, n)
            touched = torch.zeros(N, dtype=torch.bool)
            touched[reach[n]] = True
            fine = ~touched
            near(got[n][fine.to(DEV)], ref[n][fine.numpy()], rounded(n, ref, tol, i["q"].dtype)[fine.numpy()], f"{name} {n}")
        for n in ("last", "dh0"):
            assert torch.equal(got[n][1], clean[n][1]) and torch.equal(got[n][:, others], clean[n][:, others]), (name, n)
        assert torch.equal(got["dlog_decay"][others], clean["dlog_decay"][others])
        assert name != "k" or not torch.isfinite(got["o"][after, 1]).all()


@pytest.mark.parametrize("low", [-0.5, -5.0, -float("inf")])
def test_a_nan_lasts_to_its_sequence_end(low):
    """Over segments in which a state decays to nothing in 32 bits too; not into the next sequence."""
    N, at, end = 4096, 700, 3500
    i = make(N, 2, 1, 16, 24, "fp32", seed=3)
    i["v"][at, 0, 5] = float("nan")
    log_decay = torch.tensor([low, -0.01], device=DEV)
    ptr = torch.tensor([0, end, N], dtype=torch.int32, device=DEV)
    got = cpe.cp_linear_attention(i["q"], i["k"], i["v"], log_decay, seq_ptr=ptr, want_last=True)
    back = cpe.cp_linear_attention(i["q"], i["k"], i["v"], log_decay, seq_ptr=ptr, reverse=True, want_last=True)
    for out, rows in ((got, slice(at, end)), (back, slice(0, at + 1))):
        want = torch.zeros(N, 2, 24, dtype=torch.bool, device=DEV)
        want[rows, :, 5] = True
        assert torch.equal(out["o"].isnan(), want) and torch.equal(out["last"].isnan().any(2), want[[at, N - 1]])


@pytest.mark.parametrize("dtype", TYPES)
def test_decays(dtype):
    i = make(200, 6, 6, 32, 32, dtype, seed=7, h0=True, grad=True)
    i["log_decay"] = torch.tensor([0.0, -float("inf"), -1e30, -50.0, -1e-7, -0.3], device=DEV)
    check(i, [0, 200])
    # none given: 0
    a, b = (cpe.cp_linear_attention(i["q"], i["k"], i["v"], d, h0=i["h0"])["o"] for d in (None, torch.zeros(6, device=DEV)))
    assert torch.equal(a, b)
    # above 0 and NaN: their heads alone
    want = both(i)
    j = dict(i, log_decay=i["log_decay"].clone())
    j["log_decay"][2], j["log_decay"][4] = 0.1, float("nan")
    got = both(j)
    fine = [0, 1, 3, 5]
    for n in ("o", "dq", "dk", "dv"):
        assert torch.equal(got[n][:, fine], want[n][:, fine]) and torch.isnan(got[n][1:-1, [2, 4]]).all(), n


@pytest.mark.parametrize("batch", [None, 3])
def test_no_rows(batch):
    lead = (0,) if batch is None else (batch, 0)
    S = batch or 1
    z = lambda *s: torch.zeros(*lead, *s, device=DEV)  # noqa: E731
    h0, dlast = torch.randn(S, 2, 8, 8, device=DEV), torch.randn(S, 2, 8, 8, device=DEV)
    decay = torch.full((2,), -0.5, device=DEV)
    fwd = cpe.cp_linear_attention(z(2, 8), z(2, 8), z(2, 8), decay, h0=h0, want_last=True, want_carry=True)
    assert torch.equal(fwd["last"], h0) and fwd["o"].shape == (*lead, 2, 8)
    bwd = cpe.cp_linear_attention_backward(z(2, 8), z(2, 8), z(2, 8), z(2, 8), decay, fwd["carry"], dlast=dlast, h0=h0)
    assert torch.equal(bwd["dh0"], dlast) and not bwd["dlog_decay"].any()
    state = torch.randn(4, 2, 8, 8, device=DEV)
    assert cpe.cp_linear_attention_step(z(2, 8), z(2, 8), z(2, 8), state)["o"].shape == (0, 2, 8) if batch is None else True


@pytest.mark.parametrize("H,N", [(1, 5000), (2, 20011)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_long_sequences(H, N, dtype):
    check(make(N, H, H, 16, 24, dtype, seed=N, h0=True, grad=True), [0, N])


@pytest.mark.parametrize("cuts", [[0, 400, 100, 778], [5, 10, 20, 778], [0, 10, 20, 900], [0, -7, 20, 778], [-2 ** 31, 2 ** 31 - 1, 0, 778], [0, 0, 0, -1]])
def test_bad_pointers(cuts):
    i = make(778, 2, 2, 16, 16, "fp32", S=3, h0=True, grad=True)
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="seq_ptr"):
        cpe.cp_linear_attention(i["q"], i["k"], i["v"], i["log_decay"], seq_ptr=ptr, h0=i["h0"], want_last=True)
    carry = cpe.cp_linear_attention(i["q"], i["k"], i["v"], i["log_decay"], seq_ptr=ptr, want_carry=True, check_status=False)["carry"]
    with pytest.raises(ValueError, match="seq_ptr"):
        cpe.cp_linear_attention_backward(i["do"], i["q"], i["k"], i["v"], i["log_decay"], carry, seq_ptr=ptr)


def test_slots_out_of_range():
    i = make(4, 2, 2, 8, 8, "fp32")
    state = torch.randn(3, 2, 8, 8, device=DEV)
    before = state.clone()
    slots = torch.tensor([3, -1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="slot"):
        cpe.cp_linear_attention_step(i["q"], i["k"], i["v"], state, i["log_decay"], slots=slots)
    got = cpe.cp_linear_attention_step(i["q"], i["k"], i["v"], state, i["log_decay"], slots=slots, check_status=False)
    assert int(got["status"]) == 128 and not got["o"].any() and torch.equal(state, before)


def test_offsets_beyond_32_bits():
    # states of more than 2^31 elements, rows and heads as far apart
    state = torch.empty(2100, 16, 256, 256, device=DEV)
    rows = torch.tensor([0, 2099, 1023, 2050], dtype=torch.int32, device=DEV)
    i = make(4, 16, 16, 256, 256, "bf16", seed=1)
    small = torch.randn(4, 16, 256, 256, device=DEV)
    state[rows.long()] = small
    far = cpe.cp_linear_attention_step(i["q"], i["k"], i["v"], state, i["log_decay"], slots=rows)["o"]
    assert torch.equal(far, cpe.cp_linear_attention_step(i["q"], i["k"], i["v"], small, i["log_decay"])["o"]) and torch.equal(state[rows.long()], small)
    del state
    i = make(130, 2, 2, 32, 48, "bf16", seed=2, h0=True, grad=True)
    want = both(i)
    buffer = torch.zeros(130 * 2 ** 24 + 2 ** 22, dtype=torch.bfloat16, device=DEV)        # 2^31 + elements
    at = 0
    views = {}
    for n in ("q", "k", "v", "do"):
        t = i[n]
        views[n] = buffer[at:].as_strided(t.shape, (2 ** 24, 2 ** 20, 1))
        views[n].copy_(t)
        at += 64
    got = both(dict(i, **views))
    assert all(torch.equal(got[n], want[n]) for n in want)
    o = buffer[2 ** 21 + 5:].as_strided(i["do"].shape, (2 ** 24, 2 ** 20, 1))
    cpe.cp_linear_attention(views["q"], views["k"], views["v"], i["log_decay"], scale=0.25, h0=i["h0"], out={"o": o})
    assert torch.equal(o, want["o"])


@pytest.mark.parametrize("packed", [False, True])
def test_calls_in_graphs_and_on_streams(packed):
    cuts = [0, 17, 17, 1000, 2500]
    i = make(2500, 2, 1, 64, 64, "bf16", S=4 if packed else 1, seed=9, h0=True, grad=True)
    kw = dict(seq_ptr=torch.tensor(cuts, dtype=torch.int32, device=DEV) if packed else None, check_status=False)
    want = both(i, **kw)
    for _ in range(3):
        again = both(i, **kw)
        assert all(torch.equal(again[n], want[n]) for n in want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = both(i, stream=stream, **kw)
    stream.synchronize()
    assert all(torch.equal(other[n], want[n]) for n in want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, both(i, **kw)))
    for turn in range(3):
        for n in ("q", "k", "v", "do"):
            i[n].copy_(torch.randn(i[n].shape, generator=torch.Generator().manual_seed(turn)).to(i[n].dtype))
        want = both(i, **kw)
        torch.cuda.synchronize()
        for graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[n], want[n]) for n in want)


def test_a_step_follows_a_prompt():
    # the last state of a prompt, kept in a slot, and rows one by one are the rows of the whole
    N, more = 100, 7
    i = make(N + more, 3, 1, 24, 40, "fp32", seed=4)
    whole, _ = reference(i["q"], i["k"], i["v"], i["log_decay"], [0, N + more], 0.5)
    _, tol = reference(i["q"], i["k"], i["v"], i["log_decay"], [0, N + more], 0.5)
    pool = torch.zeros(5, 3, 24, 40, device=DEV)
    pool[3] = cpe.cp_linear_attention(i["q"][:N], i["k"][:N], i["v"][:N], i["log_decay"], scale=0.5, want_last=True)["last"][0]
    slots = torch.tensor([-1, 3], dtype=torch.int32, device=DEV)
    for t in range(N, N + more):
        row = [torch.stack([torch.full_like(i[n][t], float("nan")), i[n][t]]) for n in ("q", "k", "v")]
        o = cpe.cp_linear_attention_step(*row, pool, i["log_decay"], scale=0.5, slots=slots)["o"]
        assert not o[0].any()
        near(o[1], whole["o"][t], tol["o"][t] + half_step(torch.float32, whole["o"][t]), f"row {t}")


# ---- the differentiable form and the policy ------------------------------------------------------------


def leaves(i, names):
    return {n: i[n].clone().requires_grad_() for n in names}


def test_autograd_passes_on_what_the_backward_call_gives():
    cuts = [0, 9, 9, 200]
    i = make(210, 4, 2, 32, 48, "bf16", S=3, seed=11, h0=True, grad=True)
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    t = leaves(i, ("q", "k", "v", "log_decay", "h0"))
    o, last = autograd.linear_attention(*(t[n] for n in ("q", "k", "v", "log_decay")), scale=0.25, h0=t["h0"], seq_ptr=ptr, reverse=True)
    got = torch.autograd.grad([o, last], list(t.values()), [i["do"], i["dlast"]])
    want = both(i, seq_ptr=ptr, reverse=True)
    assert torch.equal(o[:200], want["o"][:200]) and not o[200:].any() and torch.equal(last, want["last"])
    for g, n in zip(got, ("dq", "dk", "dv", "dlog_decay", "dh0")):
        rows = 200 if n in ("dq", "dk", "dv") else None
        assert torch.equal(g[:rows], want[n][:rows]) and (rows is None or not g[rows:].any()), n
    # the last states alone; an expanded input
    t = leaves(i, ("k", "v"))
    _, last = autograd.linear_attention(i["q"], t["k"], t["v"], i["log_decay"])
    one = torch.autograd.grad(last.sum(), list(t.values()))
    assert all(torch.isfinite(g).all() and g.any() for g in one)
    k = i["k"][:, :1].clone().requires_grad_()
    o, _ = autograd.linear_attention(i["q"], k.expand(210, 4, 32), i["v"].repeat_interleave(2, 1), i["log_decay"])
    whole = torch.autograd.grad(o, k, i["do"])[0]
    apart = cpe.cp_linear_attention(i["q"], k.detach().expand(210, 4, 32), i["v"].repeat_interleave(2, 1), i["log_decay"], want_carry=True)
    dk = cpe.cp_linear_attention_backward(i["do"], i["q"], k.detach().expand(210, 4, 32), i["v"].repeat_interleave(2, 1), i["log_decay"], apart["carry"])["dk"]
    assert torch.allclose(whole.float(), dk.float().sum(1, keepdim=True), rtol=2.0 ** -7, atol=2.0 ** -7 * float(dk.float().abs().max()) * 4)


def test_a_gradient_in_a_graph():
    i = make(300, 2, 2, 32, 32, "bf16", seed=12, grad=True)

    def one():
        t = leaves(i, ("q", "k", "v", "log_decay"))
        o, _ = autograd.linear_attention(t["q"], t["k"], t["v"], t["log_decay"])
        return torch.autograd.grad(o, list(t.values()), i["do"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one()
    for turn in range(3):
        i["q"].copy_(torch.randn(i["q"].shape, generator=torch.Generator().manual_seed(turn)))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, one()))


def plain(policy, inputs, tokens, gain):
    """The example's policy with attention, and its loss, from their formulas, in 64 bits on the CPU."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in policy.named_parameters()}

    def unit(v):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6)

    x = inputs.cpu().double() @ p["embed"]
    n, width, heads = len(x), policy.width, policy.heads
    z = unit(x) * p["w_pre.0"]
    for i in range(policy.blocks):
        q, k, v, gate = (z @ p[f"into.{i}"]).split(width, 1)
        q, k, v = (t.view(n, heads, -1).transpose(0, 1) for t in (q, k, v))
        apart = torch.arange(n).view(-1, 1) - torch.arange(n)
        decay = torch.where(apart >= 0, torch.exp(-torch.exp(p[f"bias.{i}"]).view(-1, 1, 1) * apart.clamp(min=0)), 0.0)
        o = (((q @ k.transpose(1, 2)) * decay) @ v) * q.shape[-1] ** -0.5
        y = o.transpose(0, 1).reshape(n, width) @ p[f"back.{i}"]
        x = x + 0.5 * gate * torch.sigmoid(gate) * unit(y) * p[f"w_post.{i}"]
        z = unit(x) * p[f"w_pre.{i + 1}"]
    logits = z @ p["head"]
    lp = torch.log_softmax(logits, -1)
    (-(torch.gather(lp, 1, tokens.cpu().long()) * gain.cpu().double()).sum() + (lp.exp() * lp).sum()).backward()
    return logits.detach(), {k: v.grad for k, v in p.items()}


def test_a_policy_with_attention_against_its_formulas():
    # A stage (a product over 96 values, an operator) is off by at most some 64 steps of 2^-24 relative to its terms, there are nine of them each
    # way, and sums over rows whose terms cancel can lose a factor of ten.
    most = 10 * 2 * 9 * 64 * 2 ** -24
    w = make_workload("tiny")
    policy = example.AttentionPolicy(w.k, width=96, blocks=2, dtype=torch.float32).to(DEV)
    inputs, order = example.features(w)
    inputs = inputs.to(DEV)
    logits = policy(inputs)
    tokens = example.draw_tokens(logits.detach(), 30, top_p=0.95)
    gain = torch.randn(30, generator=torch.Generator().manual_seed(7)).to(DEV)
    logp, entropy = autograd.token_logprobs(logits, tokens)
    (-(logp * gain).sum() - entropy.sum()).backward()
    want, grads = plain(policy, inputs, tokens, gain)
    off = lambda got, ref: float((got.detach().cpu().double() - ref).norm() / ref.norm())  # noqa: E731
    assert off(logits, want) <= most
    for name, value in policy.named_parameters():
        assert off(value.grad, grads[name]) <= most, name
    # one vertex after the other, and what is drawn goes to cp_eval as it is
    states = policy.states(1, DEV)
    rows = torch.cat([policy.step(inputs[t:t + 1], states) for t in range(w.n)])
    assert off(rows, want) <= most
    graph = cpe.CpGraph.from_workload(w, device=DEV)
    assert example.rate(graph, w, order.to(DEV), tokens).shape == (30,)


def test_the_example_runs_with_attention():
    w = make_workload("tiny")
    policy, history, best = example.train(w, steps=3, partitions=40, width=64, layer="attention")
    assert len(history) == 3 and np.isfinite(history).all() and best <= max(history)
    assert all(torch.isfinite(p).all() for p in policy.parameters())
    placed = example.place(policy, w)
    assert placed.shape == (w.n,) and int(placed.max()) < w.k
