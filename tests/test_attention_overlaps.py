"""Results of cp_linear_attention, its gradient and its step that lie where an operand does are refused.  On the CPU, with made-up
addresses: a call that is not refused ends at its launch."""
import pytest
import torch

from test_attention_refusals import ATTEND, BACK, STEP
from test_policy_refusals import ARG, lib, with_  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses would be launched")

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
