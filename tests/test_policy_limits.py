"""Limits of the policy operators' entry points, on the CPU: every call here returns before anything is launched (the
addresses are made up)."""
import pytest
import torch

from test_policy_refusals import ARG, LOGP, LOGP_BACK, P, SCAN, SCAN_BACK, SIZE, lib, with_  # noqa: F401

NO_GPU = not torch.cuda.is_available()       # (elsewhere a call with made-up addresses would be launched)


def test_counts_that_end_near_the_largest_number(lib):
    # a kernel's counter goes on by up to 1,024 from the last of them, and would not pass the end but begin again below zero
    most = 0x7ffffc00
    assert lib.cp_recurrence(*with_(SCAN, ptr=P, status=P, num_seq=most + 1)) == SIZE
    assert lib.cp_recurrence_backward(*with_(SCAN_BACK, ptr=P, status=P, num_seq=most + 1)) == SIZE
    assert lib.cp_token_logprobs(*with_(LOGP, vocab=8, given=most + 1)) == SIZE
    assert lib.cp_token_logprobs_backward(*with_(LOGP_BACK, vocab=8, given=most + 1)) == SIZE
    if NO_GPU:
        assert lib.cp_recurrence(*with_(SCAN, ptr=P, status=P, num_seq=most)) != SIZE
        assert lib.cp_token_logprobs(*with_(LOGP, vocab=8, given=most)) != SIZE


@pytest.mark.parametrize("scale", [2.4e38, 2.5e38, 3.0e38, 3.4e38, float("inf"), float("nan"), -0.0, -1e-30])
def test_scales_that_are_infinite_in_units_of_ln_2(lib, scale):
    assert lib.cp_token_logprobs(*with_(LOGP, scale=scale)) == ARG
    assert lib.cp_token_logprobs_backward(*with_(LOGP_BACK, scale=scale)) == ARG


@pytest.mark.skipif(not NO_GPU, reason="the call would be launched")
@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e30, 2.3e38])
def test_scales_that_are_taken(lib, scale):
    assert lib.cp_token_logprobs(*with_(LOGP, scale=scale)) != ARG
    assert lib.cp_token_logprobs_backward(*with_(LOGP_BACK, scale=scale)) != ARG
