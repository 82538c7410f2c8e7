"""What cp_linear_attention, its gradient, its step and cp_token_sample refuse, on the CPU: every call here returns before anything is
launched (the addresses are made up).  And the 64-bit reference of the attention's GPU tests against autograd and differences."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from attention_util import reference
from paper_1711_01912_amd import attention, policy
from test_policy_refusals import ARG, NULL, SIZE, WORKSPACE, lib, with_  # noqa: F401

NO_GPU = not torch.cuda.is_available()       # (elsewhere a call with made-up addresses would be launched)


def spread(**args):
    """Every "at" becomes an address of its own, far from the others'."""
    return {k: (i + 1) << 36 if v == "at" else v for i, (k, v) in enumerate(args.items())}


ATTEND = spread(rows=256, num_seq=1, ptr=None, heads=2, kv_heads=2, wk=32, wv=64, type=1, reverse=0, q="at", ldq=64, hdq=32, k="at", ldk=64, hdk=32,
                v="at", ldv=128, hdv=64, decay="at", scale=1.0, h0=None, o="at", ldo=128, hdo=64, last="at", carry="at", work="at", bytes=1 << 30,
                stream=None, status=None)
COMMON = [(dict(type=3), ARG), (dict(type=-1), ARG), (dict(reverse=2), ARG), (dict(rows=-1), SIZE), (dict(rows=1 << 31), SIZE), (dict(num_seq=0), SIZE),
          (dict(num_seq=3), SIZE), (dict(heads=0), SIZE), (dict(heads=1025, kv_heads=1025), SIZE), (dict(heads=3), SIZE), (dict(kv_heads=0), SIZE),
          (dict(wk=0), SIZE), (dict(wk=257), SIZE), (dict(wv=0), SIZE), (dict(wv=257), SIZE), (dict(rows=1 << 30, num_seq=1 << 30), SIZE),
          (dict(ldq=-1), SIZE), (dict(hdk=-2), SIZE), (dict(ldv=(1 << 28) + 1), SIZE), (dict(hdq=(1 << 40) + 1), SIZE), (dict(q=None), NULL),
          (dict(k=None), NULL), (dict(v=None), NULL), (dict(ptr=5 << 40), NULL), (dict(work=None), NULL), (dict(work=(90 << 36) + 8), WORKSPACE),
          (dict(bytes=16), WORKSPACE)]


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(o=None), NULL), (dict(ldo=63), SIZE), (dict(hdo=63), SIZE), (dict(ldo=0), SIZE), (dict(hdo=0), SIZE), (dict(ldo=100), SIZE),
    (dict(hdo=64 * 255), SIZE), (dict(work=None, carry=None), NULL)])
def test_attention(lib, change, code):
    assert lib.cp_linear_attention(*with_(ATTEND, **change)) == code


BACK = spread(rows=256, num_seq=1, ptr=None, heads=2, kv_heads=2, wk=32, wv=64, type=1, reverse=0, do="at", lddo=128, hddo=64, dlast="at", q="at",
              ldq=64, hdq=32, k="at", ldk=64, hdk=32, v="at", ldv=128, hdv=64, decay="at", scale=1.0, h0="at", carry="at", dq="at", lddq=64, hddq=32,
              dk="at", lddk=64, hddk=32, dv="at", lddv=128, hddv=64, ddecay="at", dh0="at", work="at", bytes=1 << 30, stream=None, status=None)


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(do=None), NULL), (dict(dq=None), NULL), (dict(dk=None), NULL), (dict(dv=None), NULL), (dict(carry=None), NULL), (dict(lddq=31), SIZE),
    (dict(hddk=31), SIZE), (dict(lddv=0), SIZE), (dict(hddv=0), SIZE), (dict(lddo=-1), SIZE)])
def test_attention_backward(lib, change, code):
    assert lib.cp_linear_attention_backward(*with_(BACK, **change)) == code


STEP = spread(num_seq=5, heads=2, kv_heads=1, wk=32, wv=64, type=2, q="at", ldq=64, hdq=32, k="at", ldk=32, hdk=32, v="at", ldv=64, hdv=64, decay="at",
              scale=1.0, state="at", num_slots=8, slots="at", o="at", ldo=128, hdo=64, stream=None, status="at")


@pytest.mark.parametrize("change,code", [
    (dict(type=4), ARG), (dict(num_seq=-1), SIZE), (dict(num_slots=0), SIZE), (dict(slots=None, num_seq=9), SIZE), (dict(heads=0), SIZE),
    (dict(kv_heads=4), SIZE), (dict(wk=300), SIZE), (dict(wv=0), SIZE), (dict(ldo=127), SIZE), (dict(hdo=1), SIZE), (dict(ldq=-5), SIZE),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(o=None), NULL), (dict(state=None), NULL), (dict(status=None), NULL)])
def test_step(lib, change, code):
    assert lib.cp_linear_attention_step(*with_(STEP, **change)) == code


@pytest.mark.parametrize("entry,args,ins,outs", [
    ("cp_linear_attention", ATTEND, ("q", "k", "v", "decay"), ("o", "last", "carry", "work")),
    ("cp_linear_attention_backward", BACK, ("do", "dlast", "q", "k", "v", "decay", "h0", "carry"), ("dq", "dk", "dv", "ddecay", "dh0", "work")),
    ("cp_linear_attention_step", STEP, ("q", "k", "v", "decay", "slots"), ("o", "state", "status"))])
def test_results_where_something_else_lies(lib, entry, args, ins, outs):
    for out in outs:
        for other in ins + outs:
            if other != out:
                off = 0 if "work" in (out, other) or "status" in (out, other) else 4       # (a status is 4 bytes long)
                assert getattr(lib, entry)(*with_(args, **{out: args[other] + off})) == ARG, (out, other)
    if NO_GPU:
        assert getattr(lib, entry)(*args.values()) not in (ARG, SIZE, NULL, WORKSPACE)


@pytest.mark.skipif(not NO_GPU, reason="the calls would be launched")
def test_results_between_inputs(lib):
    # slices of one buffer [rows][heads][q k v o] and of [rows][q k v o], heads in front of rows
    P = 7 << 36
    inter = dict(rows=256, heads=2, kv_heads=2, wk=32, wv=32, ldq=256, hdq=128, ldk=256, hdk=128, ldv=256, hdv=128, ldo=256, hdo=128)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 64, v=P + 128, o=P + 192, **inter)) not in (ARG, SIZE)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 64, v=P + 128, o=P + 190, **inter)) == ARG
    fused = dict(rows=256, heads=2, kv_heads=2, wk=32, wv=32, ldq=256, hdq=32, ldk=256, hdk=32, ldv=256, hdv=32, ldo=256, hdo=32)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 128, v=P + 256, o=P + 384, **fused)) not in (ARG, SIZE)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 128, v=P + 256, o=P + 382, **fused)) == ARG
    front = dict(rows=256, heads=2, kv_heads=2, wk=32, wv=32, ldq=32, hdq=8192, ldk=32, hdk=8192, ldv=32, hdv=8192, ldo=32, hdo=8192)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 32768, v=P + 65536, o=P + 98304, **front)) not in (ARG, SIZE)
    assert lib.cp_linear_attention(*with_(ATTEND, q=P, k=P + 32768, v=P + 65536, o=P + 98302, **front)) == ARG
    # one row or head of inputs for all
    assert lib.cp_linear_attention(*with_(ATTEND, ldq=0, hdk=0)) not in (ARG, SIZE)


SAMPLE = spread(rows=8, vocab=100, type=1, logits="at", ld=100, scale=1.0, scales=None, allow=None, top_k=0, top_ks=None, top_p=1.0, top_ps=None,
                min_p=0.0, min_ps=None, given=3, u="at", urs=3, us=1, tokens="at", token_type=4, trs=3, ts=1, logp="at", work=None, bytes=0, stream=None,
                status=None)


@pytest.mark.parametrize("change,code", [
    (dict(type=3), ARG), (dict(token_type=2), ARG), (dict(scale=0.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=1e39), ARG), (dict(top_k=-1), ARG), (dict(top_p=-0.1), ARG), (dict(top_p=1.1), ARG), (dict(top_p=float("nan")), ARG),
    (dict(min_p=-0.1), ARG), (dict(min_p=1.5), ARG), (dict(min_p=float("nan")), ARG), (dict(rows=-1), SIZE), (dict(rows=1 << 31), SIZE), (dict(vocab=0), SIZE),
    (dict(vocab=(1 << 26) + 1), SIZE), (dict(given=-1), SIZE), (dict(given=0x7ffffc01), SIZE), (dict(ld=99), SIZE), (dict(token_type=1, vocab=256, ld=256), SIZE),
    (dict(trs=2), SIZE), (dict(trs=0), SIZE), (dict(ts=0), SIZE), (dict(trs=-3), SIZE), (dict(us=-1), SIZE), (dict(urs=(1 << 28) + 1), SIZE),
    (dict(ts=8, trs=2), SIZE), (dict(logits=None), NULL), (dict(u=None), NULL), (dict(tokens=None), NULL), (dict(scales=9 << 40), NULL),
    (dict(top_ks=9 << 40), NULL)])
def test_sample(lib, change, code):
    assert lib.cp_token_sample(*with_(SAMPLE, **change)) == code


def test_sample_results_where_something_else_lies(lib):
    for out in ("tokens", "logp"):
        for other in ("logits", "u", "tokens", "logp"):
            if other != out:
                assert lib.cp_token_sample(*with_(SAMPLE, **{out: SAMPLE[other] + 4})) == ARG, (out, other)
    if NO_GPU:
        # tokens of a row or of a column as neighbours, and between others
        for trs, ts in ((3, 1), (1, 8), (6, 2), (2, 16), (40, 1)):
            assert lib.cp_token_sample(*with_(SAMPLE, trs=trs, ts=ts)) not in (ARG, SIZE), (trs, ts)
        assert lib.cp_token_sample(*with_(SAMPLE, urs=0, us=0)) not in (ARG, SIZE)


def test_sample_workspace(lib):
    need, long_ = C.c_size_t(0), dict(rows=4, vocab=100000, ld=100000, logits=5 << 44, u=6 << 44, tokens=7 << 44, logp=None)
    assert lib.cp_token_sample_workspace_bytes(4, 100000, SAMPLE["given"], C.byref(need)) == 0 and need.value > 0
    for change, code in ((dict(work=None), NULL), (dict(work=(1 << 44) + 8), WORKSPACE), (dict(bytes=need.value - 1), WORKSPACE),
                         (dict(work=5 << 44), ARG), (dict(work=(7 << 44) - need.value // 512 * 256), ARG)):
        assert lib.cp_token_sample(*with_(SAMPLE, **{**long_, "work": 1 << 44, "bytes": need.value, **change})) == code, change
    assert lib.cp_token_sample_workspace_bytes(65, 100000, 1, C.byref(need)) == 0 and need.value == 0


def test_sizes(lib):
    out, states = C.c_size_t(0), C.c_int64(0)
    assert lib.cp_linear_attention_workspace_bytes(5000, 1, 1, 2, 1, 64, 64, 1, C.byref(out)) == 0 and out.value > 0
    assert lib.cp_linear_attention_workspace_bytes(5000, 1, 1, 2, 1, 64, 64, 1, None) == NULL
    assert lib.cp_linear_attention_workspace_bytes(5000, 3, 0, 2, 1, 64, 64, 1, C.byref(out)) == SIZE
    assert lib.cp_linear_attention_carry_states(5000, 1, 0, 2, 64, 64, C.byref(states)) == 0 and states.value > 1
    # a sequence that is not cut has no states to keep
    assert lib.cp_linear_attention_carry_states(5000, 5000, 0, 2, 64, 64, C.byref(states)) == 0 and states.value == 0
    assert lib.cp_linear_attention_carry_states(5000, 1, 0, 2, 64, 64, None) == NULL
    assert lib.cp_token_sample_workspace_bytes(4, 100000, 2, C.byref(out)) == 0
    assert lib.cp_token_sample_workspace_bytes(4, 100000, 2, None) == NULL
    assert lib.cp_token_sample_workspace_bytes(4, 0, 2, C.byref(out)) == SIZE


def test_constants():
    text = open(__file__.rsplit("/tests/", 1)[0] + "/include/cpeval.h").read()
    line = next(row for row in text.splitlines() if row.startswith("#define CP_STATUS_BAD_SAMPLING "))
    assert int(line.split()[2]) == policy.STATUS_BAD_SAMPLING


def test_the_binding_checks_its_tensors():
    x = torch.zeros(4, 2, 8)
    for call in (lambda: cpe.cp_linear_attention(x, x, x), lambda: cpe.cp_linear_attention_step(x, x, x, x), lambda: cpe.cp_token_sample(x[0], x[0])):
        with pytest.raises(ValueError, match="GPU"):
            call()
    h = lambda t, lead=(4,), heads=2, width=8: attention._heads(t, "t", lead, heads, width, torch.float32, t.device)[1:]  # noqa: E731
    assert h(x) == (16, 8) and h(torch.zeros(2, 4, 8).transpose(0, 1)) == (8, 32) and h(torch.zeros(4, 2, 24)[..., 8:16]) == (48, 24)
    assert h(torch.zeros(4, 1, 8).expand(4, 2, 8)) == (8, 0) and h(torch.zeros(1, 2, 8).expand(4, 2, 8)) == (0, 8)
    assert h(torch.zeros(3, 4, 2, 8), (3, 4)) == (16, 8) and h(torch.zeros(3, 1, 2, 8), (3, 1)) == (16, 8) and h(torch.zeros(1, 2, 8)[:, :1], (1,), 1) == (8, 8)
    for bad, lead in ((torch.zeros(4, 2, 16)[..., ::2], (4,)), (torch.zeros(4, 3, 8), (4,)), (torch.zeros(2, 3, 4, 8).transpose(1, 2)[:, :, :2], (2, 4)),
                      (torch.zeros(2, 6, 2, 8)[:, :4], (2, 4))):
        with pytest.raises(ValueError):
            h(bad, lead)
    with pytest.raises(TypeError):
        h(x.half())
    for q, k, v, ptr in ((x[0], x, x, None), (x, x[:, :0], x, None), (torch.zeros(4, 3, 8), x, x, None), (torch.zeros(2, 4, 2, 8),) * 3 + (torch.zeros(3, dtype=torch.int32),),
                         (x, x, x, torch.zeros(3, dtype=torch.int64))):
        with pytest.raises(ValueError):
            attention._shape(q, k, v, ptr, x.device)


# ---- the reference ----------------------------------------------------------------------------------


def problem(seed, H=4, KV=2):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    ptr = [0, 6, 6, 7, 19]
    return ptr, r(19, H, 3), r(19, KV, 3), r(19, KV, 5), -r(H).abs(), r(4, H, 3, 5), r(19, H, 5), r(4, H, 3, 5)


def forward(ptr, q, k, v, decay, h0, reverse):
    o, last = [None] * len(q), []
    k, v = (t.repeat_interleave(q.shape[1] // t.shape[1], 1) for t in (k, v))
    for s in range(len(ptr) - 1):
        state = h0[s]
        for t in reversed(range(ptr[s], ptr[s + 1])) if reverse else range(ptr[s], ptr[s + 1]):
            state = decay.exp().view(-1, 1, 1) * state + k[t].unsqueeze(-1) * v[t].unsqueeze(-2)
            o[t] = 0.3 * (q[t].unsqueeze(-1) * state).sum(-2)
        last.append(state)
    return torch.stack(o), torch.stack(last)


@pytest.mark.parametrize("reverse", [False, True])
def test_reference_against_autograd(reverse):
    ptr, q, k, v, decay, h0, do, dlast = problem(1)
    leaf = [t.clone().requires_grad_() for t in (q, k, v, decay, h0)]
    o, last = forward(ptr, *leaf, reverse)
    want = torch.autograd.grad((o * do).sum() + (last * dlast).sum(), leaf)
    out, tol = reference(q, k, v, decay, ptr, 0.3, h0, reverse, do, dlast)
    assert np.allclose(out["o"], o.detach()) and np.allclose(out["last"], last.detach())
    for key, w in zip(("dq", "dk", "dv", "dlog_decay", "dh0"), want):
        assert np.allclose(out[key], w), key
        assert out[key].shape == tol[key].shape


def test_reference_against_differences():
    ptr, *ins, do, dlast = problem(2)
    out, _ = reference(ins[0], ins[1], ins[2], ins[3], ptr, 0.3, ins[4], False, do, dlast)
    loss = lambda a: sum(float((x * d).sum()) for x, d in zip(forward(ptr, *a, False), (do, dlast)))  # noqa: E731
    g = torch.Generator().manual_seed(3)
    for i, key in enumerate(("dq", "dk", "dv", "dlog_decay", "dh0")):
        way = torch.randn(ins[i].shape, generator=g, dtype=torch.float64)
        up, down = ([t + e * way if n == i else t for n, t in enumerate(ins)] for e in (1e-6, -1e-6))
        slope = (loss(up) - loss(down)) / 2e-6
        # (a difference of steps h is off by h^2 of the third derivative and by 2^-53 / h of the value)
        assert abs(slope - float((torch.from_numpy(out[key]) * way).sum())) < 1e-6 * (1 + abs(slope)), key
