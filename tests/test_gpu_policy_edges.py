"""The operators of a learned placement policy at the borders of what their kernels divide among workgroups."""
import pytest
import torch

import paper_1711_01912_amd as cpe
import test_gpu_norm_gate as N
import test_gpu_token_logprobs as L
from policy_util import TYPES, half_step, near, recurrence

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("given", [2, 3, 40])
@pytest.mark.parametrize("rows,vocab,kind", [
    (100, 1025, "fp32"), (9, 1027, "fp32"), (300, 2051, "fp32"), (5, 4097, "fp32"), (100, 2049, "bf16"), (100, 2049, "fp16"), (9, 2055, "fp16"),
    (300, 4097, "bf16"), (600, 8193, "bf16"), (3, 65537, "bf16"), (2, 65537, "fp32"),
    (4200, 8193, "bf16"),                    # (results past the caches)
])
def test_tokens_at_places_that_begin_a_row_s_last_vector(rows, vocab, kind, given, mask):
    # the last slice of a row has fewer places than a vector: the places in front of it are those of another workgroup,
    # which adds what the tokens pass on
    d = L.make(rows, vocab, kind, given, seed=vocab, mask=mask)
    g = torch.Generator().manual_seed(given)
    d["tokens"][:, :2] = torch.randint(vocab - 8, vocab, (rows, 2), generator=g).to(DEV)
    d["tokens"][0, :2] = vocab - 4
    fwd, bwd = L.compare(d, f"{rows}x{vocab} {kind} {given} {mask}")
    allow = L.pack_mask(d["allowed"]).to(DEV) if mask else None
    for _ in range(3):
        again = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], fwd["stats"], d["dlogp"], dentropy=d["dentropy"], scale=0.8, allow=allow)
        assert torch.equal(again["dlogits"], bwd["dlogits"])


def test_more_rows_than_a_grid_s_first_dimension_has_threads_for():
    rows, vocab = 2 ** 24 + 3, 257          # a workgroup of 256 threads each: 2^32 threads and more
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    tok = torch.randint(0, vocab, (rows, 2), generator=g, device=DEV, dtype=torch.int32)
    dlogp = torch.ones(1, 2, device=DEV).expand(rows, 2)
    fwd = cpe.cp_token_logprobs(x, tok, top=2)
    grad = cpe.cp_token_logprobs_backward(x, tok, fwd["stats"], dlogp)["dlogits"]
    for lo, hi in ((0, 3), (2 ** 22 - 2, 2 ** 22 + 2), (2 ** 23 - 2, 2 ** 23 + 2), (2 ** 24 - 2, rows)):
        one = cpe.cp_token_logprobs(x[lo:hi], tok[lo:hi], top=2)
        assert all(torch.equal(fwd[k][lo:hi], one[k]) for k in ("logp", "entropy", "stats", "top_logp", "top_idx")), lo
        assert torch.equal(grad[lo:hi], cpe.cp_token_logprobs_backward(x[lo:hi], tok[lo:hi], one["stats"], dlogp[lo:hi])["dlogits"]), lo


def test_the_gradient_of_as_many_rows_as_there_may_be():
    # 2^23 tiles of 512 threads: as many threads as a dimension of a grid may not have
    rows = 2 ** 31 - 1
    g = torch.Generator(device=DEV).manual_seed(6)
    f, x, dh = (torch.empty(rows, 1, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(3))
    cuts = [0, 700, rows - 900, rows]
    ptr = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    dlast = torch.randn(3, 1, generator=g, device=DEV)
    fwd = cpe.cp_recurrence(f, x, seq_ptr=ptr, want_last=True, want_carry=True)
    bwd = cpe.cp_recurrence_backward(dh, f, x, fwd["carry"], seq_ptr=ptr, dlast=dlast)
    got = {"h": fwd["h"], "df": bwd["df"], "dx": bwd["dx"]}
    for i, (lo, hi) in enumerate(((0, 700), (0, 0), (rows - 900, rows))):
        if lo == hi:
            continue
        ref, tol = recurrence(f[lo:hi], x[lo:hi], [0, hi - lo], dh=dh[lo:hi], dlast=dlast[i:i + 1])
        for key, t in got.items():
            near(t[lo:hi], ref[key], tol[key] + half_step(t.dtype, ref[key]), f"rows from {lo} {key}")
        near(fwd["last"][i], ref["last"][0], tol["last"][0] + half_step(torch.float32, ref["last"][0]), f"last {i}")


@pytest.mark.parametrize("scale", [1e-30, 1e30, 2.3e38])
def test_scales_from_end_to_end(scale):
    for vocab in (9, 4000):
        L.compare(L.make(4, vocab, "fp32", 3, seed=vocab), f"{vocab} {scale}", scale=scale, top=3)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("rows,width,kind", [(700, 1111, "fp16"), (300, 4101, "bf16"), (40, 5003, "fp32"), (9, 16381, "bf16"), (1000, 70, "bf16"), (200, 301, "fp16"), (50, 5, "fp32")])
def test_outputs_of_a_joint_in_the_place_of_its_inputs(rows, width, kind, post):
    d = N.make(rows, width, kind, kind, seed=width)
    kw = dict(w_pre=d["w_pre"], w_post=d["w_post"] if post else None, scale=0.5)
    fwd = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], want_stats=True, **kw)
    bwd = cpe.cp_norm_gate_backward(d["dr"], d["dz"], d["x"], d["y"], d["gate"], stats=fwd["stats"], **kw)
    for r, z in (("x", "y"), ("y", "gate"), ("gate", "x"), ("x", None), (None, "x")):
        c = {k: d[k].clone() for k in ("x", "y", "gate")}
        got = cpe.cp_norm_gate(c["x"], c["y"], c["gate"], out={k: c[v] for k, v in (("r", r), ("z", z)) if v}, **kw)
        assert torch.equal(got["r"], fwd["r"]) and torch.equal(got["z"], fwd["z"]), (r, z)
    for dx, dy, dgate in (("x", "y", "gate"), ("dr", "dz", "x"), ("y", "x", "dr")):
        c = {k: d[k].clone() for k in ("x", "y", "gate", "dr", "dz")}
        got = cpe.cp_norm_gate_backward(c["dr"], c["dz"], c["x"], c["y"], c["gate"], stats=fwd["stats"],
                                        out={"dx": c[dx], "dy": c[dy], "dgate": c[dgate]}, **kw)
        assert all(torch.equal(got[k], bwd[k]) for k in bwd), (dx, dy, dgate)


def test_a_step_in_the_place_of_its_input():
    for width in (64, 67):
        g = torch.Generator().manual_seed(width)
        f, x, state = (torch.randn(50, width, generator=g).to(DEV) for _ in range(3))
        want_state = state.clone()
        want = cpe.cp_recurrence_step(f, x, want_state)["h"]
        for over in (0, 1):
            st, fx = state.clone(), [f.clone(), x.clone()]
            assert torch.equal(cpe.cp_recurrence_step(*fx, st, out={"h": fx[over]})["h"], want) and torch.equal(st, want_state)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,given", [(3000, 5, 9), (3000, 13, 100), (1000, 64, 30), (777, 200, 300), (300, 256, 1)])
def test_a_gradient_in_the_place_of_few_logits(rows, vocab, given, kind):
    d = L.make(rows, vocab, kind, given, seed=vocab, mask=True)
    allow = L.pack_mask(d["allowed"]).to(DEV)
    stats = cpe.cp_token_logprobs(d["logits"], d["tokens"], allow=allow)["stats"]
    want = cpe.cp_token_logprobs_backward(d["logits"], d["tokens"], stats, d["dlogp"], dentropy=d["dentropy"], allow=allow)["dlogits"]
    x = d["logits"].clone()
    cpe.cp_token_logprobs_backward(x, d["tokens"], stats, d["dlogp"], dentropy=d["dentropy"], allow=allow, out={"dlogits": x})
    assert torch.equal(x, want)


def test_results_over_inputs_that_are_read_again_are_refused():
    x = torch.randn(300, 300, device=DEV)
    with pytest.raises(cpe.CpError):
        cpe.cp_recurrence(x, x.clone(), out={"h": x})
    fwd = cpe.cp_recurrence(x, x, want_last=True, want_carry=True)
    with pytest.raises(cpe.CpError):
        cpe.cp_recurrence_backward(x.clone(), x, x, fwd["carry"], out={"df": x})
    with pytest.raises(cpe.CpError):
        cpe.cp_recurrence(x, x, h0=fwd["last"], want_last=True, out={"last": fwd["last"]})
    got = cpe.cp_token_logprobs(x)
    with pytest.raises(cpe.CpError):
        cpe.cp_token_logprobs_backward(x, None, got["stats"], None, dentropy=got["entropy"], out={"dlogits": x})


def test_checked_calls_on_the_current_and_on_another_stream():
    x = torch.randn(64, 8, device=DEV)
    tok, ptr = torch.full((64, 3), 2, device=DEV), torch.tensor([0, 9, 64], dtype=torch.int32, device=DEV)
    state, slots = torch.zeros(64, 8, device=DEV), torch.arange(64, dtype=torch.int32, device=DEV)
    bad_tok, bad_ptr, bad_slots = torch.full_like(tok, 8), torch.flip(ptr, [0]), slots + 1
    torch.cuda.synchronize()
    for stream in (None, torch.cuda.Stream(), None):
        for _ in range(20):
            cpe.cp_token_logprobs(x, tok, stream=stream)
            cpe.cp_recurrence(x, x, seq_ptr=ptr, stream=stream)
            cpe.cp_recurrence_step(x, x, state, slots=slots, stream=stream)
            for call in (lambda: cpe.cp_token_logprobs(x, bad_tok, stream=stream), lambda: cpe.cp_recurrence(x, x, seq_ptr=bad_ptr, stream=stream),
                         lambda: cpe.cp_recurrence_step(x, x, state, slots=bad_slots, stream=stream)):
                with pytest.raises(ValueError):
                    call()
        torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [9, 64, 200, 300, 1401, 2100, 4000, 40000])
def test_a_nan_is_no_alternative_and_hides_none(vocab, kind):
    # quiet and signalling, beside the best places of their vectors, in front of and behind them
    top = min(vocab, 20)
    g = torch.Generator().manual_seed(vocab)
    dt = TYPES[kind]
    bits = torch.int32 if kind == "fp32" else torch.int16
    quiet, signalling = {"fp32": (0x7fc00000, 0x7f800001), "bf16": (0x7fc0, 0x7f81), "fp16": (0x7e00, 0x7c01)}[kind]
    x = (torch.randn(6, vocab, generator=g) * 2.5).to(dt)
    best = torch.sort(x, dim=-1, descending=True, stable=True).indices
    for row, (word, step) in enumerate(((quiet, 1), (quiet, -1), (signalling, 1), (signalling, -1), (quiet, 3), (signalling, 2))):
        at = (best[row, [0, 1, 3]] + step) % vocab
        x[row].view(bits)[at] = word if word < 2 ** 15 or kind == "fp32" else word - 2 ** 16
    got = cpe.cp_token_logprobs(x.to(DEV), top=top)
    assert got["entropy"].isnan().all() and got["top_logp"][got["top_idx"] >= 0].isnan().all()
    for row in range(6):
        order = torch.where(x[row].isnan(), float("-inf"), x[row].float())
        want = torch.sort(order, dim=-1, descending=True, stable=True).indices[:top]
        want = torch.where(order[want] == float("-inf"), -1, want)
        assert got["top_idx"][row].tolist() == want.tolist(), row


@pytest.mark.parametrize("width", [8193, 9001, 16383, 16384])
@pytest.mark.parametrize("block,stream", [("fp32", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
def test_the_widest_rows_of_a_joint(width, block, stream):
    N.compare(N.make(300, width, block, stream, seed=width), f"{width} {block} {stream}")
    N.compare(N.make(3, width, block, stream, weights="fp32", seed=3), f"{width} {block} {stream}, without", gate=False, post=False, dr=False)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab,given,ints", [(40, 8, 64, torch.uint8), (33, 16, 257, torch.int32), (7, 50, 1000, torch.int64), (300, 4, 12, torch.uint8),
                                                   (11, 2, 1024, torch.int32), (70, 45, 113, torch.uint8), (9, 200, 300, torch.int64), (5, 256, 1000, torch.uint8)])
def test_many_tokens_of_few_places_in_16_bits(rows, vocab, given, ints, kind):
    L.compare(L.make(rows, vocab, kind, given, seed=given, ints=ints, mask=True), f"{rows} {vocab} {given} {kind}")


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,given", [(9, 3), (9, 40), (64, 3), (200, 100), (300, 1), (300, 3), (4000, 2), (20001, 1)])
def test_what_has_no_probability_gets_no_gradient(vocab, given, kind):
    # whatever flows into its row: a row without a place has an entropy of 0, by which a loss may have divided
    d = L.make(8, vocab, kind, given, seed=vocab, mask=True)
    d["allowed"][3] = False
    d["allowed"][7] = True
    allow, open_ = L.pack_mask(d["allowed"]).to(DEV), torch.from_numpy(d["allowed"]).to(DEV)
    x, dlogp, de = d["logits"].clone(), d["dlogp"].clone(), d["dentropy"].clone()
    x[7, 1::2] = float("-inf")
    d["tokens"][5:8, 0] = torch.from_numpy(d["allowed"][5:8].argmax(1)).to(DEV)
    de[3], de[4], de[6] = float("inf"), float("nan"), float("-inf")         # rows 3 and 4 have no place
    dlogp[5, 0], dlogp[7, 0] = float("inf"), float("nan")
    x[2, int(d["allowed"][2].argmax())] = float("nan")
    stats = cpe.cp_token_logprobs(x, d["tokens"], allow=allow)["stats"]
    g = cpe.cp_token_logprobs_backward(x, d["tokens"], stats, dlogp, dentropy=de, allow=allow)["dlogits"]
    none = ~open_ | (x == float("-inf"))
    assert (g[none] == 0).all()
    assert g[2][~none[2]].isnan().all() and g[7][~none[7]].isnan().all() and not g[5][~none[5]].isfinite().all()
    assert g[[0, 1]].isfinite().all() and not (~none[[3, 4]]).any()


def test_rows_that_lie_beyond_2_to_the_31_elements():
    rows, ld, width = 270000, 8200, 72
    buf = torch.zeros(rows, ld, dtype=torch.bfloat16, device=DEV)        # 2.2e9 elements
    g = torch.Generator(device=DEV).manual_seed(9)
    v = {k: torch.randn(rows, width, generator=g, device=DEV).bfloat16() for k in ("f", "x", "dh")}
    cut = {k: buf[:, 1 + 100 * i:1 + 100 * i + width] for i, k in enumerate(("f", "x", "dh", "h", "df", "dx", "dgate", "gone"))}
    for key, t in v.items():
        cut[key].copy_(t)
    bias, w = torch.linspace(0, 4, width, device=DEV), torch.ones(width, dtype=torch.bfloat16, device=DEV)
    tok = torch.randint(0, width, (rows, 1), generator=g, device=DEV, dtype=torch.int32)
    for reverse in (False, True):
        a = cpe.cp_recurrence(v["f"], v["x"], bias=bias, reverse=reverse, want_carry=True, want_last=True)
        b = cpe.cp_recurrence(cut["f"], cut["x"], bias=bias, reverse=reverse, want_carry=True, want_last=True, out={"h": cut["h"]})
        assert torch.equal(a["h"], b["h"]) and torch.equal(a["last"], b["last"]) and torch.equal(a["carry"], b["carry"])
        c = cpe.cp_recurrence_backward(v["dh"], v["f"], v["x"], a["carry"], bias=bias, reverse=reverse)
        d = cpe.cp_recurrence_backward(cut["dh"], cut["f"], cut["x"], a["carry"], bias=bias, reverse=reverse, out={k: cut[k] for k in ("df", "dx")})
        assert all(torch.equal(c[k], d[k]) for k in ("df", "dx", "dbias"))
    a = cpe.cp_norm_gate(v["x"], v["f"], v["dh"], w_pre=w, w_post=w, want_stats=True)
    b = cpe.cp_norm_gate(cut["x"], cut["f"], cut["dh"], w_pre=w, w_post=w, want_stats=True, out={"r": cut["df"], "z": cut["dx"]})
    assert all(torch.equal(a[k], b[k]) for k in ("r", "z", "stats"))
    c = cpe.cp_norm_gate_backward(None, v["dh"], v["x"], v["f"], v["dh"], w_pre=w, w_post=w, stats=a["stats"])
    d = cpe.cp_norm_gate_backward(None, cut["dh"], cut["x"], cut["f"], cut["dh"], w_pre=w, w_post=w, stats=a["stats"],
                                  out={"dx": cut["dx"], "dy": cut["df"], "dgate": cut["dgate"]})
    assert all(torch.equal(c[k], d[k]) for k in c)
    a, b = cpe.cp_token_logprobs(v["x"], tok, top=3), cpe.cp_token_logprobs(cut["x"], tok, top=3)
    assert all(torch.equal(a[k], b[k]) for k in a)
    c = cpe.cp_token_logprobs_backward(v["x"], tok, a["stats"], a["logp"], dentropy=a["entropy"])["dlogits"]
    d = cpe.cp_token_logprobs_backward(cut["x"], tok, a["stats"], a["logp"], dentropy=a["entropy"], out={"dlogits": cut["h"]})["dlogits"]
    assert torch.equal(c, d) and not cut["gone"].any()
    x = torch.randn(rows, 1000, generator=g, device=DEV).bfloat16()
    wide, tok = buf[:, 3:1003], tok * 13
    wide.copy_(x)
    a, b = cpe.cp_token_logprobs(x, tok, top=3), cpe.cp_token_logprobs(wide, tok, top=3)
    assert all(torch.equal(a[k], b[k]) for k in a)
    c = cpe.cp_token_logprobs_backward(x, tok, a["stats"], a["logp"], dentropy=a["entropy"])["dlogits"]
    d = cpe.cp_token_logprobs_backward(wide, tok, a["stats"], a["logp"], dentropy=a["entropy"], out={"dlogits": buf[:, 2001:3001]})["dlogits"]
    assert torch.equal(c, d) and not buf[:, 3001:].any()
