"""Which results of cp_linear_attention, its gradient and its step lie where an operand does, against the bytes themselves: calls that share
any are refused, and results between the rows and heads of inputs that are as far apart are not.  On the CPU, with made-up
addresses: a call that is not refused ends at its launch."""
import random

import pytest
import torch

from test_attention_refusals import ATTEND, BACK, STEP
from test_policy_refusals import ARG, NULL, SIZE, WORKSPACE, lib, with_  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses would be launched")
P = 7 << 36


def one_row(**more):
    return dict(rows=1, num_seq=1, **more)


@pytest.mark.parametrize("off", [2, 4, 8, 16, 32, 64, 126, -2, -62, -126, 0])
def test_one_row(lib, off):
    # bf16, two heads of 64: 256 bytes each
    size = dict(heads=2, kv_heads=2, wk=64, wv=64)
    for name in "qkv":
        assert lib.cp_linear_attention_step(*with_(STEP, num_seq=1, type=1, ldq=128, hdq=64, ldk=128, hdk=64, ldv=128, hdv=64, ldo=128, hdo=64, **size,
                                                   o=STEP[name] + off)) == ARG, name
        assert lib.cp_linear_attention(*with_(ATTEND, **one_row(ldq=128, hdq=64, ldk=128, hdk=64, ldv=128, hdv=64, ldo=128, hdo=64, **size),
                                              o=ATTEND[name] + off)) == ARG, name
    back = one_row(lddo=128, hddo=64, ldq=128, hdq=64, ldk=128, hdk=64, ldv=128, hdv=64, lddq=128, hddq=64, lddk=128, hddk=64, lddv=128, hddv=64, **size)
    for out in ("dq", "dk", "dv"):
        for name in ("do", "q", "k", "v", "dq", "dk", "dv"):
            if name != out:
                assert lib.cp_linear_attention_backward(*with_(BACK, **back, **{out: BACK[name] + off})) == ARG, (out, name)


def bytes_of(at, ld, hd, rows, heads, width, each):
    return {at + (r * ld + h * hd + c) * each + b for r in range(rows) for h in range(heads) for c in range(width) for b in range(each)}


@pytest.mark.parametrize("seed", range(40))
def test_a_few_rows_against_their_bytes(lib, seed):
    g = random.Random(seed)
    met = apart = 0
    for _ in range(100):
        rows, kv, group = g.choice([1, 1, 2, 3, 5]), g.choice([1, 2]), g.choice([1, 2])
        heads, wk, wv, each = kv * group, g.randint(1, 6), g.randint(1, 6), g.choice([2, 4])
        # a result whose rows and heads lie apart, an input with the same distances
        if g.random() < 0.5:
            hd = wv + g.randint(0, 3)
            ld = (heads - 1) * hd + wv + g.randint(0, 9)
        else:
            ld = wv + g.randint(0, 3)
            hd = (rows - 1) * ld + wv + g.randint(0, 9)
        name = g.choice(["q", "v"])
        n, w = (heads, wk) if name == "q" else (kv, wv)
        off = each * g.randint(-((rows - 1) * ld + heads * hd + 8), (rows - 1) * ld + heads * hd + 8)
        far = dict(q=1 << 40, k=2 << 40, v=3 << 40, o=P, state=5 << 40, decay=None, slots=None, status=None, num_slots=8)
        far[name] = P + off
        change = dict(num_seq=rows, heads=heads, kv_heads=kv, wk=wk, wv=wv, type=0 if each == 4 else 1, ldq=ld, hdq=hd, ldk=16, hdk=8, ldv=ld, hdv=hd, ldo=ld, hdo=hd, **far)
        share = bool(bytes_of(P, ld, hd, rows, heads, wv, each) & bytes_of(P + off, ld, hd, rows, n, w, each))
        met, apart = met + share, apart + (not share)
        code = lib.cp_linear_attention_step(*with_(STEP, **change))
        assert (code == ARG) == share and code not in (SIZE, NULL, WORKSPACE), (change, name, off, code)
    assert met > 10 and apart > 10
