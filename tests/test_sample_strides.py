"""Strides that cp_token_sample does not use: of a single row, of a single draw.  On the CPU, with made-up addresses: a call that is not refused
ends at its launch."""
import pytest
import torch

from test_attention_refusals import SAMPLE
from test_policy_refusals import ARG, SIZE, lib, with_  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses would be launched")


@pytest.mark.parametrize("change", [dict(rows=1, urs=1 << 40), dict(rows=1, trs=1 << 40), dict(rows=1, urs=-3, trs=0), dict(given=1, us=1 << 40), dict(given=1, ts=1 << 40),
                                    dict(given=1, us=-1, ts=-1), dict(rows=1, given=1, urs=-1, trs=-1, us=-1, ts=-1),
                                    # one row of more draws than a stride may be
                                    dict(rows=1, given=1 << 29, urs=1 << 29, trs=1 << 29)])
def test_unused(lib, change):
    assert lib.cp_token_sample(*with_(SAMPLE, **change)) not in (ARG, SIZE)


@pytest.mark.parametrize("change", [dict(urs=(1 << 28) + 1), dict(trs=(1 << 28) + 1), dict(us=(1 << 28) + 1), dict(ts=(1 << 28) + 1), dict(us=-1), dict(urs=-1), dict(ts=0), dict(trs=0)])
def test_used(lib, change):
    assert lib.cp_token_sample(*with_(SAMPLE, **change)) == SIZE


@pytest.mark.parametrize("rows,given", [(1, 5), (5, 1), (1, 1)])
def test_results_over_inputs(lib, rows, given):
    # int32 tokens and logp in the place of the numbers, whatever the unused strides say
    far = dict(rows=rows, given=given, urs=1 if given == 1 else 1 << 40, us=1 << 40 if given == 1 else 1, trs=1 if given == 1 else 1 << 40, ts=1 << 40 if given == 1 else 1)
    for out in ("tokens", "logp"):
        for off in range(0, 4 * rows * given, 4):
            assert lib.cp_token_sample(*with_(SAMPLE, **far, **{out: SAMPLE["u"] + off})) == ARG, (out, off)
        assert lib.cp_token_sample(*with_(SAMPLE, **far, **{out: SAMPLE["u"] + 4 * rows * given})) not in (ARG, SIZE)
