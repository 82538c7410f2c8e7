"""Limits of the policy operators' entry points, on the CPU: every call here returns before anything is launched (the
addresses are made up)."""
import pytest
import torch

from paper_1711_01912_amd import policy
from test_policy_refusals import ARG, LOGP, LOGP_BACK, NORM, NORM_BACK, P, SCAN, SCAN_BACK, SIZE, STEP, lib, with_  # noqa: F401

NO_GPU = not torch.cuda.is_available()       # (elsewhere a call with made-up addresses would be launched)


def apart(args, **there):
    """The arguments with every array at an address of its own, far from the others', and those of `there` too."""
    got = {k: P + (i << 32) if v == P and isinstance(v, int) else v for i, (k, v) in enumerate(args.items())}
    assert all(k in got for k in there)
    return {**got, **{k: P + (i + 100 << 32) for i, k in enumerate(there) if there[k] is None}, **{k: v for k, v in there.items() if v is not None}}


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
    assert lib.cp_token_logprobs(*with_(apart(LOGP), scale=scale)) != ARG
    assert lib.cp_token_logprobs_backward(*with_(apart(LOGP_BACK), scale=scale)) != ARG


# ---- results where something else lies ------------------------------------------------------------------

ALL = [("cp_recurrence", apart(SCAN, bias=None, h0=None, last=None, carry=None)),
       ("cp_recurrence_backward", apart(SCAN_BACK, dlast=None, bias=None, h0=None, dbias=None, dh0=None)),
       ("cp_recurrence_step", apart(STEP, bias=None, slots=None, status=None)),
       ("cp_norm_gate", apart({**NORM, "stream_type": 1}, stats=None)),
       ("cp_norm_gate_backward", apart({**NORM_BACK, "stream_type": 1})),
       ("cp_token_logprobs", apart(LOGP)),
       ("cp_token_logprobs_backward", apart({**LOGP_BACK, "vocab": 300, "ld": 300, "ldd": 300}))]
BY_NAME = dict(ALL)
IN = {"cp_recurrence": ("f", "x", "bias", "h0"), "cp_recurrence_backward": ("dh", "f", "x", "dlast", "bias", "h0", "carry"),
      "cp_recurrence_step": ("f", "x", "bias", "slots"), "cp_norm_gate": ("x", "y", "gate", "w_pre", "w_post"),
      "cp_norm_gate_backward": ("dr", "dz", "x", "y", "gate", "w_pre", "w_post", "stats"), "cp_token_logprobs": ("logits",),
      "cp_token_logprobs_backward": ("logits", "stats")}
OUT = {"cp_recurrence": ("h", "last", "carry"), "cp_recurrence_backward": ("df", "dx", "dbias", "dh0"), "cp_recurrence_step": ("state", "h"),
       "cp_norm_gate": ("r", "z", "stats"), "cp_norm_gate_backward": ("dx", "dy", "dgate", "dw_pre", "dw_post"),
       "cp_token_logprobs": ("logp", "entropy", "stats", "top_logp", "top_idx"), "cp_token_logprobs_backward": ("dlogits",)}
# (a result that may take an input's place, and those whose gradient sums are formed in a launch of their own)
FINE = {("cp_recurrence_step", "h", "f"), ("cp_recurrence_step", "h", "x")}
FINE |= {("cp_norm_gate", o, i) for o in ("r", "z") for i in ("x", "y", "gate")}
FINE |= {("cp_norm_gate_backward", o, i) for o in ("dx", "dy", "dgate") for i in ("dr", "dz", "x", "y", "gate")}
FINE |= {("cp_norm_gate_backward", o, i) for o in ("dw_pre", "dw_post") for i in ("w_pre", "w_post")}


@pytest.mark.skipif(not NO_GPU, reason="the call would be launched")
@pytest.mark.parametrize("name,args", ALL)
def test_results_apart_from_everything_are_taken(lib, name, args):
    assert getattr(lib, name)(*args.values()) not in (ARG, SIZE, -1, -9)


@pytest.mark.parametrize("name,out,other", [(n, o, i) for n in OUT for o in OUT[n] for i in IN[n] + OUT[n] if o != i])
def test_results_where_something_else_lies_are_refused(lib, name, out, other):
    args = BY_NAME[name]
    for off in (0, 2):
        if off == 0 and (name, out, other) in FINE:
            if NO_GPU:
                assert getattr(lib, name)(*with_(args, **{out: args[other]})) != ARG
        elif not (name, out, other) in FINE or not out.startswith("dw"):
            assert getattr(lib, name)(*with_(args, **{out: args[other] + off})) == ARG, off


@pytest.mark.skipif(not NO_GPU, reason="the calls would be launched")
def test_slices_of_one_buffer_lie_between_each_other(lib):
    scan = {**BY_NAME["cp_recurrence"], "ldf": 200, "ldx": 200, "ldh": 200}        # bf16: 400 bytes a row, 128 of each slice
    f = scan["f"]
    for x, h, fine in ((128, 256, True), (272, 128, True), (256, 126, False), (128, 254, False), (128, 274, False), (128, 400 + 256, True),
                       (128, 400 * 255 + 100, False), (128, 400 * 255 + 256, True), (128, -400 * 256 + 256, True), (128, -400 + 272, True),
                       (128, -400 + 274, False), (128, 400 * 256 + 10, True), (128, 400 * 255 + 128, False), (400 * 256, 128, True)):
        got = lib.cp_recurrence(*with_(scan, x=f + x, h=f + h))
        assert (got != ARG) == fine, (x, h)
    # rows that are unequally far apart lie somewhere among each other
    assert lib.cp_recurrence(*with_(scan, h=f + 128, ldh=199)) == ARG
    assert lib.cp_recurrence(*with_(scan, h=f + 400 * 256, ldh=199)) != ARG
    one = {**BY_NAME["cp_recurrence"], "rows": 1}                                   # a single row has no distance
    assert lib.cp_recurrence(*with_(one, h=one["f"] + 128)) != ARG and lib.cp_recurrence(*with_(one, h=one["f"] + 126)) == ARG


def test_places_of_other_types_and_of_few_logits(lib):
    norm = {**BY_NAME["cp_norm_gate"], "stream_type": 0}                            # x and r of 32 bits, y and z of 16
    assert lib.cp_norm_gate(*with_(norm, z=norm["x"])) == ARG and lib.cp_norm_gate(*with_(norm, r=norm["y"])) == ARG
    grad = BY_NAME["cp_token_logprobs_backward"]
    if NO_GPU:
        assert lib.cp_norm_gate(*with_(norm, z=norm["y"])) != ARG and lib.cp_norm_gate(*with_(norm, r=norm["x"])) != ARG
        assert lib.cp_token_logprobs_backward(*with_(grad, vocab=256, dlogits=grad["logits"])) != ARG
    assert lib.cp_token_logprobs_backward(*with_(grad, vocab=257, dlogits=grad["logits"])) == ARG
    assert lib.cp_token_logprobs_backward(*with_(grad, vocab=256, dlogits=grad["logits"], ldd=299)) == ARG


# ---- the binding ----------------------------------------------------------------------------------------


def test_a_status_is_waited_for_on_its_stream_alone(monkeypatch):
    def never(*args):
        raise AssertionError("waits for every stream of the device")

    class Stream:
        waits = 0

        def synchronize(self):
            self.waits += 1

    monkeypatch.setattr(torch.cuda, "synchronize", never)
    stream, told, fine = Stream(), torch.tensor([32], dtype=torch.int32), torch.tensor([64], dtype=torch.int32)
    with pytest.raises(ValueError, match="bad"):
        policy._check(told, policy.STATUS_BAD_TOKEN, "bad", stream)
    policy._check(fine, policy.STATUS_BAD_TOKEN, "bad", stream)
    policy._check(fine, policy.STATUS_BAD_TOKEN, "bad", None)
    assert stream.waits == 2


def test_rows_of_several_axes_are_equally_far_apart():
    m = lambda t, rows, width: policy._matrix(t, "t", rows, width, torch.float32, t.device)  # noqa: E731
    t = torch.zeros(2, 3, 5, 20)
    assert m(t, 30, 20) == 20 and m(t[..., 3:11], 30, 8) == 20
    assert m(t[:1, :, :, :8], 15, 8) == 20 and m(t[:1, :1, :, :8], 5, 8) == 20
    assert m(t[:, :, 2:3, :8], 6, 8) == 100 and m(t[:, 1:2, 2:3, :8], 2, 8) == 300 and m(t[1:, 1:2, 2:3, :8], 1, 8) == 8
    assert m(torch.zeros(4, 1, 7, 6)[..., :4], 28, 4) == 6
    for bad, rows, width in ((t[:, :2], 20, 20), (t[:, :, :4], 24, 20), (t[:, :2, :, :8], 20, 8), (t.transpose(0, 1), 30, 20),
                             (t.transpose(1, 2)[..., :8], 30, 8), (t[:, :, ::2, :8], 18, 8), (torch.zeros(3, 5, 20).expand(2, 3, 5, 20), 30, 20),
                             (torch.zeros(2, 3, 1, 8).expand(2, 3, 5, 8), 30, 8)):
        with pytest.raises(ValueError):
            m(bad, rows, width)
