"""The differentiable functions and the example that trains a placement policy with them."""
import os
import sys

import pytest
import torch

import paper_1711_01912_amd as cpe
from workloads import make_workload

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import learn_placement as example  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def leaf(*shape, seed, dtype=torch.float32):
    return randn(*shape, seed=seed, dtype=dtype).requires_grad_()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_recurrence_passes_on_what_the_backward_call_gives(dtype):
    from paper_1711_01912_amd import autograd
    fused = leaf(300, 3 * 40, seed=0, dtype=dtype)
    bias, h0 = leaf(40, seed=1), leaf(3, 40, seed=2)
    ptr = torch.tensor([0, 11, 11, 300], dtype=torch.int32, device=DEV)
    f, x, _ = fused.split(40, 1)
    h, last = autograd.recurrence(f, x, bias=bias, h0=h0, seq_ptr=ptr, reverse=True)
    dh, dlast = randn(300, 40, seed=3, dtype=dtype), randn(3, 40, seed=4)
    got = torch.autograd.grad([h, last], [fused, bias, h0], [dh, dlast])
    with torch.no_grad():
        kw = dict(bias=bias, h0=h0, seq_ptr=ptr, reverse=True)
        fwd = cpe.cp_recurrence(f, x, want_carry=True, want_last=True, **kw)
        want = cpe.cp_recurrence_backward(dh, f, x, fwd["carry"], dlast=dlast, **kw)
    assert torch.equal(h, fwd["h"]) and torch.equal(last, fwd["last"])
    assert torch.equal(got[0][:, :40], want["df"]) and torch.equal(got[0][:, 40:80], want["dx"]) and not got[0][:, 80:].any()
    assert torch.equal(got[1], want["dbias"]) and torch.equal(got[2], want["dh0"])
    # an expanded gradient, of one output alone
    h, last = autograd.recurrence(f, x, bias=bias, h0=h0, seq_ptr=ptr, reverse=True)
    one = torch.autograd.grad(last.sum(), [fused, h0])
    want = cpe.cp_recurrence_backward(torch.zeros_like(dh), f.detach(), x.detach(), fwd["carry"], dlast=torch.ones_like(dlast), bias=bias.detach(),
                                      h0=h0.detach(), seq_ptr=ptr, reverse=True)
    assert torch.equal(one[0][:, :40], want["df"]) and torch.equal(one[1], want["dh0"])


def test_norm_gate_passes_on_what_the_backward_call_gives():
    from paper_1711_01912_amd import autograd
    x, y, gate = leaf(37, 96, seed=0), leaf(37, 96, seed=1, dtype=torch.bfloat16), leaf(37, 96, seed=2, dtype=torch.bfloat16)
    w_pre, w_post = leaf(96, seed=3), leaf(96, seed=4)
    dr, dz = randn(37, 96, seed=5), randn(37, 96, seed=6, dtype=torch.bfloat16)
    kw = dict(w_pre=w_pre, w_post=w_post, gate_act="silu", scale=0.5)
    r, z = autograd.norm_gate(x, y, gate, **kw)
    got = torch.autograd.grad([r, z], [x, y, gate, w_pre, w_post], [dr, dz])
    with torch.no_grad():
        fwd = cpe.cp_norm_gate(x, y, gate, want_stats=True, **kw)
        want = cpe.cp_norm_gate_backward(dr, dz, x, y, gate, stats=fwd["stats"], **kw)
    assert torch.equal(r, fwd["r"]) and torch.equal(z, fwd["z"])
    assert all(torch.equal(g, want[k]) for g, k in zip(got, ("dx", "dy", "dgate", "dw_pre", "dw_post")))
    # without a block: the stream goes by
    r, z = autograd.norm_gate(x, w_pre=w_pre, z_dtype=torch.bfloat16)
    assert r is x
    one = torch.autograd.grad([r, z], [x], [dr, dz])[0]
    with torch.no_grad():
        fwd = cpe.cp_norm_gate(x, w_pre=w_pre, z_dtype=torch.bfloat16, want_stats=True)
        want = cpe.cp_norm_gate_backward(None, dz, x, w_pre=w_pre, stats=fwd["stats"])
    assert torch.equal(one, want["dx"] + dr)


def test_token_logprobs_pass_on_what_the_backward_call_gives():
    from paper_1711_01912_amd import autograd
    logits = leaf(50, 9, seed=0)
    tokens = torch.randint(0, 9, (50, 40), generator=torch.Generator().manual_seed(1)).to(torch.uint8).to(DEV)
    weights, de = randn(40, seed=2).expand(50, 40), randn(50, seed=3)
    logp, entropy = autograd.token_logprobs(logits, tokens, scale=0.7)
    got = torch.autograd.grad([logp, entropy], [logits], [weights, de])[0]
    with torch.no_grad():
        fwd = cpe.cp_token_logprobs(logits, tokens, scale=0.7)
        want = cpe.cp_token_logprobs_backward(logits, tokens, fwd["stats"], weights, dentropy=de, scale=0.7)
        alone = cpe.cp_token_logprobs_backward(logits, None, fwd["stats"], None, dentropy=torch.ones_like(de), scale=0.7)
    assert torch.equal(logp, fwd["logp"]) and torch.equal(entropy, fwd["entropy"]) and torch.equal(got, want["dlogits"])
    _, entropy = autograd.token_logprobs(logits, tokens, scale=0.7)
    assert torch.equal(torch.autograd.grad(entropy.sum(), [logits])[0], alone["dlogits"])


def plain(policy, inputs, tokens, gain):
    """The example's policy and loss from its formulas, in 64 bits on the CPU."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in policy.named_parameters()}

    def unit(v):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6)

    x, width = inputs.cpu().double() @ p["embed"], policy.width
    z = unit(x) * p["w_pre.0"]
    for i in range(policy.blocks):
        f, v, gate = (z @ p[f"into.{i}"]).split(width, 1)
        a = torch.sigmoid(f + p[f"bias.{i}"])
        rows, h = [], torch.zeros(width, dtype=torch.float64)
        for t in range(len(a)):
            h = a[t] * h + (1 - a[t]) * v[t]
            rows.append(h)
        y = torch.stack(rows) @ p[f"back.{i}"]
        x = x + 0.5 * gate * torch.sigmoid(gate) * unit(y) * p[f"w_post.{i}"]
        z = unit(x) * p[f"w_pre.{i + 1}"]
    logits = z @ p["head"]
    lp = torch.log_softmax(logits, -1)
    loss = -(torch.gather(lp, 1, tokens.cpu().long()) * gain.cpu().double()).sum() + (lp.exp() * lp).sum()
    loss.backward()
    return logits.detach(), {k: v.grad for k, v in p.items()}


def test_policy_against_its_formulas():
    # A stage (a product over 96 values, an operator) is off by at most some 64 steps of 2^-24 relative to its terms, there are
    # nine of them each way, and sums over rows whose terms cancel can lose a factor of ten.
    most = 10 * 2 * 9 * 64 * 2 ** -24
    from paper_1711_01912_amd import autograd
    w = make_workload("tiny")
    policy = example.Policy(w.k, width=96, blocks=2, dtype=torch.float32).to(DEV)
    inputs = example.features(w)[0].to(DEV)
    logits = policy(inputs)
    tokens, gain = example.draw(logits.detach(), 30), randn(30, seed=7)
    logp, entropy = autograd.token_logprobs(logits, tokens)
    (-(logp * gain).sum() - entropy.sum()).backward()
    want, grads = plain(policy, inputs, tokens, gain)
    off = lambda got, ref: float((got.detach().cpu().double() - ref).norm() / ref.norm())  # noqa: E731
    assert off(logits, want) <= most
    for name, value in policy.named_parameters():
        assert off(value.grad, grads[name]) <= most, name
    # one vertex after the other
    states = torch.zeros(2, 1, 96, device=DEV)
    rows = torch.cat([policy.step(inputs[t:t + 1], states) for t in range(w.n)])
    assert off(rows, want) <= most


def test_training_shortens_critical_paths():
    w = make_workload("tiny")
    policy, history, best = example.train(w, steps=60, partitions=128, width=64, blocks=2)
    assert sum(history[-5:]) < 0.95 * sum(history[:5])
    placed = example.place(policy, w)
    assert placed.shape == (w.n,) and int(placed.max()) < w.k
    graph = cpe.CpGraph.from_workload(w, device=DEV)
    assert float(cpe.cp_eval(graph, placed.view(1, -1), w.speeds, w.bandwidth)["cp"][0]) < history[0]


def test_a_training_pass_in_a_graph():
    from paper_1711_01912_amd import autograd
    fused, w_pre, w_post = randn(200, 3 * 64, seed=0), randn(64, seed=1), randn(64, seed=2)
    tokens = torch.randint(0, 64, (200, 3), generator=torch.Generator().manual_seed(3)).to(DEV)

    def one(fused):
        fused = fused.detach().requires_grad_()
        f, x, gate = fused.split(64, 1)
        h, _ = autograd.recurrence(f, x)
        r, z = autograd.norm_gate(x, h, gate, w_pre=w_pre, w_post=w_post)
        logp, entropy = autograd.token_logprobs(z, tokens)
        # (weights made without a library's sum over many blocks)
        return torch.autograd.grad([r, logp, entropy], [fused], [torch.ones_like(r), torch.ones_like(logp), torch.ones_like(entropy)])[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one(fused)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one(fused)
    for turn in range(4):
        fused.copy_(randn(200, 3 * 64, seed=10 + turn))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, one(fused))
