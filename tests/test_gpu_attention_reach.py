"""What a NaN or an infinity in one row of cp_linear_attention has to reach, element by element, and what pointers that do not rise must
not reach: memory around the results."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from attention_util import reference
from policy_util import wide
from test_gpu_linear_attention import make, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run(i, out=None, back=None, **kw):
    kw = dict(scale=0.25, h0=i["h0"], **kw)
    got = cpe.cp_linear_attention(i["q"], i["k"], i["v"], i["log_decay"], want_last=True, want_carry=True, out=out, **kw)
    got.update(cpe.cp_linear_attention_backward(i["do"], i["q"], i["k"], i["v"], i["log_decay"], got["carry"], dlast=i["dlast"], out=back, **kw))
    return got


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,K,V", [("fp32", 32, 32), ("bf16", 64, 128), ("bf16", 128, 128), ("fp16", 40, 48), ("bf16", 256, 64), ("fp32", 7, 33)])
def test_what_is_no_number_arrives(dtype, K, V, bad, reverse):
    # every element that the formula makes infinite or NaN, in 64 bits and with the same values, is neither finite here, and all others are what
    # they are
    N, H, cuts = 300, 3, [0, 250, 300]
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    i = make(N, H, H, K, V, dtype, S=2, seed=6, h0=True, grad=True)
    for name in ("q", "k", "v", "do"):
        for at in (0, 133, 249):
            j = dict(i, **{name: i[name].clone()})
            j[name][at, 1, 2] = bad
            got = run(j, seq_ptr=ptr, reverse=reverse)
            ref, tol = reference(j["q"], j["k"], j["v"], j["log_decay"], cuts, 0.25, j["h0"], reverse, j["do"], j["dlast"])
            some = 0
            for n in ("o", "last", "dq", "dk", "dv", "dh0", "dlog_decay"):
                odd = ~np.isfinite(ref[n])
                some += int(odd.sum())
                value, fine = wide(got[n]).reshape(odd.shape), np.where(odd, 0.0, ref[n])
                lost = odd & np.isfinite(value)
                assert not lost.any(), (name, at, n, np.argwhere(lost)[:3].tolist())
                with np.errstate(invalid="ignore"):
                    off = np.abs(value - fine) <= np.where(odd, 0.0, rounded(n, {n: fine}, tol, i["q"].dtype))
                assert (off | odd).all(), (name, at, n, np.argwhere(~(off | odd))[:3].tolist())
            assert some > 0


def middle(shape, dtype, value, guard=1 << 16):
    """(a tensor inside a larger buffer, the buffer's rest is as it was)"""
    size = int(np.prod(shape))
    room = torch.full((guard + size + guard,), value, dtype=dtype, device=DEV)
    return room[guard:guard + size].view(shape), lambda: bool((room[:guard] == value).all()) and bool((room[guard + size:] == value).all())


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype,K,V", [("fp32", 16, 16), ("bf16", 64, 96)])
@pytest.mark.parametrize("cuts", [[0, 400, 100, 778], [5, 10, 20, 778], [0, 10, 20, 900], [0, -7, 20, 778], [-2 ** 31, 2 ** 31 - 1, 0, 778], [0, 0, 0, -1],
                                  [778, 778, 778, 778], [0, 900, 900, 778], [2 ** 31 - 1] * 4])
def test_bad_pointers_write_inside_the_results(cuts, dtype, K, V, reverse):
    N, H, S = 778, 2, 3
    i = make(N, H, 1, K, V, dtype, S=S, h0=True, grad=True)
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    dt, state = i["q"].dtype, (S, H, K, V)
    shapes = dict(o=((N, H, V), dt), last=(state, torch.float32)), dict(dq=((N, H, K), dt), dk=((N, 1, K), dt), dv=((N, 1, V), dt), dh0=(state, torch.float32),
                                                                      dlog_decay=((H,), torch.float32))
    fwd, back = ({n: middle(*s, 7.0) for n, s in part.items()} for part in shapes)
    got = run(i, {n: t for n, (t, _) in fwd.items()}, {n: t for n, (t, _) in back.items()}, seq_ptr=ptr, reverse=reverse, check_status=False)
    assert int(got["status"]) == 64
    for n, (_, untouched) in {**fwd, **back}.items():
        assert untouched(), n
