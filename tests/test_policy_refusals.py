"""What the entry points of the policy's operators refuse, on the CPU: every call here returns before anything is launched
(the addresses are made up).  And the 64-bit references of their GPU tests against autograd."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from paper_1711_01912_amd import policy
from policy_util import joint, logprobs, recurrence

ARG, SIZE, NULL, WORKSPACE = -12, -2, -1, -9
P = 1 << 20          # an address, aligned


@pytest.fixture(scope="module")
def lib():
    from paper_1711_01912_amd.build import build_library
    build_library(force=False)
    return cpe.load_library()


def with_(args, **change):
    got = dict(args)
    assert all(k in got for k in change)
    got.update(change)
    return got.values()


SCAN = dict(rows=256, width=64, num_seq=1, ptr=None, type=1, reverse=0, f=P, ldf=64, x=P, ldx=64, bias=None, h0=None, h=P, ldh=64,
            last=None, carry=None, work=P, bytes=1 << 30, stream=None, status=None)


@pytest.mark.parametrize("change,code", [
    (dict(type=3), ARG), (dict(type=-1), ARG), (dict(reverse=2), ARG), (dict(rows=-1), SIZE), (dict(rows=1 << 31), SIZE),
    (dict(width=0), SIZE), (dict(width=65537), SIZE), (dict(num_seq=0), SIZE), (dict(num_seq=3), SIZE), (dict(ldf=63), SIZE),
    (dict(ldx=0), SIZE), (dict(ldh=-64), SIZE), (dict(f=None), NULL), (dict(x=None), NULL), (dict(h=None), NULL),
    (dict(ptr=P), NULL), (dict(work=None), NULL), (dict(work=P + 8), WORKSPACE), (dict(bytes=16), WORKSPACE),
])
def test_recurrence(lib, change, code):
    assert lib.cp_recurrence(*with_(SCAN, **change)) == code


SCAN_BACK = dict(rows=256, width=64, num_seq=1, ptr=None, type=1, reverse=0, dh=P, lddh=64, dlast=None, f=P, ldf=64, x=P, ldx=64,
                 bias=None, h0=None, carry=P, df=P, lddf=64, dx=P, lddx=64, dbias=None, dh0=None, work=P, bytes=1 << 30, stream=None,
                 status=None)


@pytest.mark.parametrize("change,code", [
    (dict(type=9), ARG), (dict(rows=-5), SIZE), (dict(width=-1), SIZE), (dict(num_seq=7), SIZE), (dict(lddh=1), SIZE),
    (dict(lddf=63), SIZE), (dict(lddx=63), SIZE), (dict(dh=None), NULL), (dict(carry=None), NULL), (dict(df=None), NULL),
    (dict(dx=None), NULL), (dict(ptr=P), NULL), (dict(work=None), NULL), (dict(work=P + 4), WORKSPACE), (dict(bytes=1024), WORKSPACE),
    (dict(rows=5, dbias=P, work=None), NULL),
])
def test_recurrence_backward(lib, change, code):
    assert lib.cp_recurrence_backward(*with_(SCAN_BACK, **change)) == code


STEP = dict(num_seq=4, width=64, type=0, f=P, ldf=64, x=P, ldx=64, bias=None, state=P, num_slots=4, slots=None, h=P, ldh=64, stream=None,
            status=None)


@pytest.mark.parametrize("change,code", [
    (dict(type=5), ARG), (dict(num_seq=-1), SIZE), (dict(num_seq=5), SIZE), (dict(num_slots=0), SIZE), (dict(width=0), SIZE),
    (dict(ldf=2), SIZE), (dict(state=None), NULL), (dict(f=None), NULL), (dict(h=None), NULL), (dict(slots=P), NULL),
])
def test_step(lib, change, code):
    assert lib.cp_recurrence_step(*with_(STEP, **change)) == code


NORM = dict(rows=8, width=64, stream_type=1, type=1, weight_type=1, act=1, x=P, ldx=64, y=P, ldy=64, gate=P, ldg=64, w_pre=P, w_post=P,
            scale=1.0, eps=1e-6, r=P, ldr=64, z=P, ldz=64, stats=None, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(stream_type=2), ARG), (dict(type=4), ARG), (dict(weight_type=-1), ARG), (dict(act=3), ARG), (dict(act=-1), ARG),
    (dict(y=None), ARG), (dict(rows=-1), SIZE), (dict(width=0), SIZE), (dict(width=16385), SIZE), (dict(ldx=63), SIZE),
    (dict(ldz=1), SIZE), (dict(ldg=0), SIZE), (dict(w_pre=None), NULL), (dict(x=None), NULL), (dict(z=None), NULL), (dict(r=None), NULL),
])
def test_norm_gate(lib, change, code):
    assert lib.cp_norm_gate(*with_(NORM, **change)) == code


NORM_BACK = dict(rows=8, width=64, stream_type=0, type=1, weight_type=1, act=1, dr=P, lddr=64, dz=P, lddz=64, x=P, ldx=64, y=P, ldy=64,
                 gate=P, ldg=64, w_pre=P, w_post=P, scale=1.0, stats=P, dx=P, lddx=64, dy=P, lddy=64, dgate=P, lddg=64, dw_pre=P,
                 dw_post=P, work=P, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(stream_type=2), ARG), (dict(act=7), ARG), (dict(y=None), ARG), (dict(rows=-1), SIZE), (dict(width=20000), SIZE),
    (dict(lddr=8), SIZE), (dict(lddy=8), SIZE), (dict(w_pre=None), NULL), (dict(gate=None), NULL), (dict(w_post=None), NULL),
    (dict(dz=None), NULL), (dict(stats=None), NULL), (dict(dx=None), NULL), (dict(dy=None), NULL), (dict(work=None), NULL),
    (dict(work=P + 128), WORKSPACE), (dict(bytes=100), WORKSPACE),
])
def test_norm_gate_backward(lib, change, code):
    assert lib.cp_norm_gate_backward(*with_(NORM_BACK, **change)) == code


LOGP = dict(rows=8, vocab=100, type=1, logits=P, ld=100, scale=1.0, allow=None, given=2, tokens=P, token_type=4, trs=2, ts=1, logp=P,
            entropy=P, stats=P, top=3, top_logp=P, top_idx=P, work=P, bytes=1 << 30, stream=None, status=P)


@pytest.mark.parametrize("change,code", [
    (dict(type=7), ARG), (dict(token_type=2), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG),
    (dict(scale=float("inf")), ARG), (dict(rows=-1), SIZE), (dict(vocab=0), SIZE), (dict(vocab=(1 << 26) + 1), SIZE),
    (dict(given=-1), SIZE), (dict(top=65), SIZE), (dict(top=-1), SIZE), (dict(ld=99), SIZE), (dict(logits=None), NULL),
    (dict(tokens=None), NULL), (dict(logp=None), NULL), (dict(entropy=None), NULL), (dict(stats=None), NULL), (dict(top_idx=None), NULL),
    (dict(status=None), NULL), (dict(work=P + 16), WORKSPACE),
])
def test_token_logprobs(lib, change, code):
    assert lib.cp_token_logprobs(*with_(LOGP, **change)) == code


LOGP_BACK = dict(rows=8, vocab=100, type=1, logits=P, ld=100, scale=1.0, allow=None, given=2, tokens=P, token_type=4, trs=2, ts=1,
                 stats=P, dlogp=P, drs=2, ds=1, de=None, des=0, dlogits=P, ldd=100, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(type=7), ARG), (dict(token_type=0), ARG), (dict(scale=0.0), ARG), (dict(rows=-1), SIZE), (dict(vocab=0), SIZE),
    (dict(given=-2), SIZE), (dict(ldd=99), SIZE), (dict(logits=None), NULL), (dict(stats=None), NULL), (dict(dlogp=None), NULL),
    (dict(dlogits=None), NULL), (dict(tokens=None), NULL),
])
def test_token_logprobs_backward(lib, change, code):
    assert lib.cp_token_logprobs_backward(*with_(LOGP_BACK, **change)) == code


def test_workspaces(lib):
    out = C.c_size_t(0)
    for call, good, bad in ((lib.cp_recurrence_workspace_bytes, (1000, 64, 1), (-1, 64, 0)),
                            (lib.cp_norm_gate_backward_workspace_bytes, (1000, 64), (10, 0)),
                            (lib.cp_token_logprobs_workspace_bytes, (4, 100000, 20), (4, 100, 65))):
        assert call(*good, C.byref(out)) == 0 and out.value > 0
        assert call(*good, None) == NULL
        assert call(*bad, C.byref(out)) == SIZE


def test_constants():
    text = open(__file__.rsplit("/tests/", 1)[0] + "/include/cpeval.h").read()
    for name, value in (("CP_RECURRENCE_CHUNK", policy.RECURRENCE_CHUNK), ("CP_TYPE_BF16", policy.TYPE_BF16), ("CP_TYPE_F16", policy.TYPE_F16),
                        ("CP_GATE_SIGMOID", policy.GATE_SIGMOID), ("CP_GATE_SILU", policy.GATE_SILU),
                        ("CP_STATUS_BAD_TOKEN", policy.STATUS_BAD_TOKEN), ("CP_STATUS_BAD_SEQUENCE", policy.STATUS_BAD_SEQUENCE),
                        ("CP_STATUS_BAD_SLOT", policy.STATUS_BAD_SLOT)):
        line = next(row for row in text.splitlines() if row.startswith(f"#define {name} "))
        assert int(line.split()[2]) == value, name


def test_the_binding_checks_its_tensors():
    x = torch.zeros(4, 8)
    for call in (lambda: cpe.cp_recurrence(x, x), lambda: cpe.cp_recurrence_step(x, x, x), lambda: cpe.cp_norm_gate(x, w_pre=x[0]),
                 lambda: cpe.cp_token_logprobs(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    m = lambda t, rows=4, width=8, dt=torch.float32: policy._matrix(t, "t", rows, width, dt, t.device)  # noqa: E731
    assert m(x) == 8 and m(torch.zeros(4, 20)[:, 3:11]) == 20 and m(torch.zeros(2, 2, 8)) == 8
    assert m(torch.zeros(1, 99)[:, :8], rows=1) == 8 and m(torch.zeros(0, 8), rows=0) == 8
    for bad in (torch.zeros(8, 4).t(), torch.zeros(4, 9), torch.zeros(3, 8), torch.zeros(1, 8).expand(4, 8),
                torch.zeros(2, 4, 8)[:, :2], torch.zeros(4, 16)[:, ::2]):
        with pytest.raises(ValueError):
            m(bad)
    with pytest.raises(TypeError):
        m(x.half())
    with pytest.raises(ValueError):
        policy._vector(torch.zeros(9), "v", (8,), torch.float32, x.device)
    with pytest.raises(TypeError):
        policy._vector(torch.zeros(8).half(), "v", (8,), torch.float32, x.device)
    with pytest.raises(TypeError):
        policy._type(torch.zeros(1, dtype=torch.int32), "t")


# ---- the references ----------------------------------------------------------------------------------


def test_reference_recurrence_against_autograd():
    g = torch.Generator().manual_seed(0)
    ptr = [0, 7, 7, 8, 20]
    f, x, h0, bias = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((20, 3), (20, 3), (4, 3), (3,)))
    dh, dlast = torch.randn(20, 3, generator=g, dtype=torch.float64), torch.randn(4, 3, generator=g, dtype=torch.float64)
    for reverse in (False, True):
        leaf = [t.clone().requires_grad_() for t in (f, x, h0, bias)]
        h, last = [None] * 20, []
        for s in range(4):
            state = leaf[2][s]
            for t in reversed(range(ptr[s], ptr[s + 1])) if reverse else range(ptr[s], ptr[s + 1]):
                a = torch.sigmoid(leaf[0][t] + leaf[3])
                state = a * state + (1 - a) * leaf[1][t]
                h[t] = state
            last.append(state)
        loss = (torch.stack(h) * dh).sum() + (torch.stack(last) * dlast).sum()
        want = torch.autograd.grad(loss, leaf)
        out, _ = recurrence(f, x, ptr, bias=bias, h0=h0, reverse=reverse, dh=dh, dlast=dlast)
        assert np.allclose(out["h"], torch.stack(h).detach()) and np.allclose(out["last"], torch.stack(last).detach())
        for key, w in zip(("df", "dx", "dh0", "dbias"), want):
            assert np.allclose(out[key], w), key


def test_reference_joint_against_autograd():
    g = torch.Generator().manual_seed(1)
    x, y, gate, dr, dz = (torch.randn(5, 6, generator=g, dtype=torch.float64) for _ in range(5))
    w_pre, w_post = torch.rand(6, generator=g, dtype=torch.float64), torch.rand(6, generator=g, dtype=torch.float64)
    acts = {"none": lambda t: t, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu}
    for act, fn in acts.items():
        leaf = [t.clone().requires_grad_() for t in (x, y, gate, w_pre, w_post)]
        u = leaf[1] / (leaf[1].pow(2).mean(-1, keepdim=True) + 1e-3).sqrt() * leaf[4]
        r = leaf[0] + 0.3 * fn(leaf[2]) * u
        z = r / (r.pow(2).mean(-1, keepdim=True) + 1e-3).sqrt() * leaf[3]
        want = torch.autograd.grad((r * dr).sum() + (z * dz).sum(), leaf)
        out, _ = joint(x, y, gate, w_pre, w_post, act, 0.3, 1e-3, dr=dr, dz=dz)
        for key, w in zip(("dx", "dy", "dgate", "dw_pre", "dw_post"), want):
            assert np.allclose(out[key], w), (act, key)


def test_reference_logprobs_against_autograd():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4, 9, generator=g, dtype=torch.float64)
    tok = torch.randint(0, 9, (4, 6), generator=g)
    dl, de = torch.randn(4, 6, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    leaf = x.clone().requires_grad_()
    lp = torch.log_softmax(0.7 * leaf, -1)
    ent = -(lp.exp() * lp).sum(-1)
    want = torch.autograd.grad((lp.gather(1, tok) * dl).sum() + (ent * de).sum(), leaf)[0]
    out, _ = logprobs(x, tok, 0.7, None, 3, dl, de)
    assert np.allclose(out["dlogits"], want) and np.allclose(out["logp"], lp.gather(1, tok).detach()) and np.allclose(out["entropy"], ent.detach())
    assert np.array_equal(out["top_idx"], x.topk(3).indices.numpy())
