"""cp_token_logprobs and its gradient against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from policy_util import TYPES, half_step, logprobs, near, pack_mask, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(rows, vocab, kind, given, *, seed=0, ints=torch.int64, mask=False, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=g) * spread).to(TYPES[kind])
    tok = torch.randint(0, vocab, (rows, given), generator=g)
    if given and ints != torch.uint8:
        tok[torch.rand(rows, given, generator=g) < 0.15] = -1
    allowed = None
    if mask:
        allowed = (torch.rand(rows, vocab, generator=g) < 0.6).numpy()
        allowed[rows // 2] = False
    return dict(logits=x.to(DEV), tokens=tok.to(ints).to(DEV), allowed=allowed, dlogp=torch.randn(rows, given, generator=g).to(DEV),
                dentropy=(0.3 * torch.randn(rows, generator=g)).to(DEV))


def compare(d, what, *, scale=0.8, top=0, dentropy=True):
    allow = pack_mask(d["allowed"]).to(DEV) if d["allowed"] is not None else None
    de = d["dentropy"] if dentropy else None
    ref, tol = logprobs(d["logits"], d["tokens"], scale, d["allowed"], top, d["dlogp"], de)
    fwd = cpe.cp_token_logprobs(d["logits"], d["tokens"], scale=scale, allow=allow, top=top)
    near(fwd["logp"], ref["logp"], tol["logp"] + half_step(torch.float32, ref["logp"]), what + " logp")
    near(fwd["entropy"], ref["entropy"], tol["entropy"], what + " entropy")
    if top:
        assert np.array_equal(fwd["top_idx"].cpu().numpy(), ref["top_idx"]), what
        fin = np.isfinite(ref["top_logp"])
        near(fwd["top_logp"], ref["top_logp"], np.where(fin, 2 ** -24 * (200 + 8 * np.abs(np.where(fin, ref["top_logp"], 0))), 0), what + " top")
    bwd = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], fwd["stats"], d["dlogp"], dentropy=de, scale=scale, allow=allow)
    g = bwd["dlogits"]
    near(g, ref["dlogits"], tol["dlogits"] + half_step(g.dtype, ref["dlogits"]), what + " dlogits")
    return fwd, bwd


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (5, 2), (3, 7), (66, 16), (4, 64), (9, 65), (3, 1000), (2, 2048), (5, 5003), (2, 40000)])
def test_sizes_and_types(rows, vocab, kind):
    compare(make(rows, vocab, kind, 1, seed=vocab), f"{rows}x{vocab} {kind}", top=min(vocab, 5))


@pytest.mark.parametrize("vocab", [3, 64, 130, 3000, 20001])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_masks_and_rows_without_a_place(vocab, kind):
    compare(make(7, vocab, kind, 4, seed=vocab, mask=True), f"mask {vocab}", top=8)


@pytest.mark.parametrize("ints", [torch.uint8, torch.int32, torch.int64])
@pytest.mark.parametrize("rows,vocab,given", [(1, 2, 1), (40, 8, 64), (33, 16, 257), (7, 50, 1000), (5, 200, 31), (64, 3, 5), (300, 4, 12)])
def test_many_tokens_of_few_places(rows, vocab, given, ints):
    compare(make(rows, vocab, "fp32", given, seed=given, ints=ints), f"{rows} {vocab} {given}")


@pytest.mark.parametrize("top", [1, 7, 20, 64])
def test_alternatives_with_ties(top):
    # few distinct values: ties everywhere, the lowest places first; one row of a single value
    for vocab in (5, 64, 3000, 70000):
        d = make(3, vocab, "bf16", 1, seed=top)
        d["logits"] = (d["logits"] * 2).round() / 2
        d["logits"][1] = 1.25
        d["logits"][2, : vocab // 2] = -0.0
        d["logits"][2, vocab // 2:] = 0.0
        compare(d, f"ties {vocab}", top=top)


def test_lowest_values_and_infinities():
    for kind in ("fp32", "bf16", "fp16"):
        low = torch.finfo(TYPES[kind]).min
        for vocab in (6, 70, 5000):
            d = make(5, vocab, kind, 2, seed=3)
            d["tokens"][:] = torch.tensor([0, vocab - 1])
            x = d["logits"]
            x[0] = low                          # a row of the lowest value: all places alike
            x[1, 1:] = low                      # all but one
            x[2, ::2] = float("-inf")
            x[3] = float("-inf")                # nothing
            x[4, 0] = 80.0
            for scale in (0.5, 1.0, 3.0):
                compare(d, f"{kind} {vocab} {scale}", scale=scale, top=3)


def test_nan_and_inf_spoil_their_row_alone():
    for vocab in (9, 4000):
        d = make(4, vocab, "fp32", 1, seed=8)
        want, gwant = compare(d, "clean")
        x = d["logits"].clone()
        x[1, 3] = float("nan")
        x[2, 5] = float("inf")
        got = cpe.cp_token_logprobs(x, d["tokens"].clamp(min=0), scale=0.8)
        assert got["logp"][1:3].isnan().all() and got["entropy"][1:3].isnan().all()
        assert torch.equal(got["entropy"][[0, 3]], want["entropy"][[0, 3]])
        g = cpe.cp_token_logprobs_backward(x, d["tokens"], got["stats"], d["dlogp"], dentropy=d["dentropy"], scale=0.8)["dlogits"]
        assert torch.equal(g[[0, 3]], gwant["dlogits"][[0, 3]]) and g[1].isnan().all()
        # at a place that is not allowed they are not looked at
        allowed = np.ones((4, vocab), bool)
        allowed[1, 3] = allowed[2, 5] = False
        d["logits"], d["allowed"] = x, allowed
        compare({**d, "logits": torch.where(torch.from_numpy(allowed).to(DEV), x, x)}, "masked", top=4)


def test_strides_and_broadcast_weights():
    d = make(50, 24, "bf16", 40, seed=2, ints=torch.uint8)
    buf = torch.zeros(50, 64, dtype=torch.bfloat16, device=DEV)
    for lo in (0, 8, 3):
        buf[:, lo:lo + 24] = d["logits"]
        view = buf[:, lo:lo + 24]
        turned = d["tokens"].t().contiguous().t()          # partition-major assignments, seen from the vertices
        weights = torch.randn(40, generator=torch.Generator().manual_seed(1)).to(DEV)
        a = cpe.cp_token_logprobs(d["logits"], d["tokens"])
        b = cpe.cp_token_logprobs(view, turned)
        near(b["logp"], wide(a["logp"]), 1e-5)
        ga = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], a["stats"], weights.expand(50, 40).contiguous())["dlogits"]
        room = torch.full((50, 64), 3.0, dtype=torch.bfloat16, device=DEV)
        gb = cpe.cp_token_logprobs_backward(view, turned, b["stats"], weights.expand(50, 40), dentropy=torch.zeros(1, device=DEV).expand(50),
                                            out={"dlogits": room[:, lo:lo + 24]})["dlogits"]
        near(gb, wide(ga), half_step(torch.bfloat16, wide(ga)) * 2 + 1e-5)
        assert (room[:, :lo] == 3).all() and (room[:, lo + 24:] == 3).all()
    one = cpe.cp_token_logprobs(d["logits"], d["tokens"][:, 7])
    assert one["logp"].shape == (50,) and torch.equal(one["logp"], cpe.cp_token_logprobs(d["logits"], d["tokens"])["logp"][:, 7])


def test_without_tokens_or_entropy_gradient():
    d = make(6, 300, "fp32", 1)
    alone = cpe.cp_token_logprobs(d["logits"], top=4)
    both = cpe.cp_token_logprobs(d["logits"], d["tokens"], top=4)
    assert "logp" not in alone and torch.equal(alone["entropy"], both["entropy"]) and torch.equal(alone["top_idx"], both["top_idx"])
    compare(d, "no entropy", dentropy=False)


def test_gradient_against_differences():
    d = make(6, 11, "fp32", 5, seed=5, mask=True)
    allow = pack_mask(d["allowed"]).to(DEV)
    tok = d["tokens"].cpu().numpy()
    fine = (tok >= 0) & np.take_along_axis(d["allowed"], np.maximum(tok, 0), 1)
    fwd = cpe.cp_token_logprobs(d["logits"], d["tokens"], scale=0.8, allow=allow)
    g = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], fwd["stats"], d["dlogp"], dentropy=d["dentropy"], scale=0.8, allow=allow)["dlogits"]
    base = d["logits"].double().cpu()

    def loss(x):
        out, _ = logprobs(x, d["tokens"], 0.8, d["allowed"])
        return (np.where(fine, out["logp"], 0) * wide(d["dlogp"])).sum() + (out["entropy"] * wide(d["dentropy"])).sum()

    gen = torch.Generator().manual_seed(7)
    for _ in range(3):
        way = torch.randn(base.shape, generator=gen, dtype=torch.float64)
        diff = (loss(base + 1e-5 * way) - loss(base - 1e-5 * way)) / 2e-5
        terms = g.double().cpu() * way
        assert abs(diff - terms.sum().item()) <= 2e-6 * terms.abs().sum().item() + 1e-6


def test_bad_tokens_are_told():
    for vocab in (10, 3000):
        d = make(4, vocab, "fp32", 3)
        d["tokens"][2, 1] = vocab
        with pytest.raises(ValueError):
            cpe.cp_token_logprobs(d["logits"], d["tokens"])
        got = cpe.cp_token_logprobs(d["logits"], d["tokens"], check_status=False)
        torch.cuda.synchronize()
        assert got["logp"][2, 1] == 0 and int(got["status"]) == 32
        g = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], got["stats"], d["dlogp"])["dlogits"]
        d["tokens"][2, 1] = -1
        assert torch.equal(g, cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], got["stats"], d["dlogp"])["dlogits"])


def test_no_rows():
    x = torch.zeros(0, 64, device=DEV)
    got = cpe.cp_token_logprobs(x, torch.zeros(0, 2, dtype=torch.int32, device=DEV), top=3)
    assert got["logp"].shape == (0, 2) and got["top_idx"].shape == (0, 3)
    assert cpe.cp_token_logprobs_backward(x, None, got["stats"], None, dentropy=torch.zeros(0, device=DEV))["dlogits"].shape == (0, 64)


def test_in_a_graph():
    for vocab, given in ((16, 100), (9000, 1)):
        d = make(64, vocab, "bf16", given, ints=torch.int32)
        x = d["logits"].clone()
        cpe.cp_token_logprobs(x, d["tokens"], top=4)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a = cpe.cp_token_logprobs(x, d["tokens"], top=4, check_status=False)
            b = cpe.cp_token_logprobs_backward(x, d["tokens"], a["stats"], d["dlogp"], dentropy=d["dentropy"])
        for turn in range(3):
            x.copy_(d["logits"] * (1 + turn))
            graph.replay()
            torch.cuda.synchronize()
            e = cpe.cp_token_logprobs(x, d["tokens"], top=4)
            eb = cpe.cp_token_logprobs_backward(x, d["tokens"], e["stats"], d["dlogp"], dentropy=d["dentropy"])
            assert torch.equal(a["logp"], e["logp"]) and torch.equal(a["top_idx"], e["top_idx"]) and torch.equal(b["dlogits"], eb["dlogits"])


@pytest.mark.parametrize("vocab,top", [(257, 64), (363, 1), (520, 64), (1401, 20), (2049, 33), (6000, 64), (66000, 20)])
@pytest.mark.parametrize("kind,mask", [("bf16", False), ("fp32", False), ("fp32", True)])
def test_alternatives_of_rows_that_do_not_fill_a_workgroup(vocab, top, kind, mask):
    compare(make(3, vocab, kind, 1, seed=vocab, mask=mask), f"{vocab} {top} {kind} {mask}", top=top)


@pytest.mark.parametrize("rows,vocab,given", [(70, 45, 113), (9, 64, 16), (35, 33, 20), (50, 12, 17), (50, 8, 33), (3, 64, 300), (11, 2, 1024), (9, 200, 300),
                                              (5, 256, 1000), (70, 128, 64), (20, 255, 50)])
def test_columns_of_few_tokens(rows, vocab, given):
    compare(make(rows, vocab, "fp32", given, seed=given, mask=True), f"{rows} {vocab} {given}")
