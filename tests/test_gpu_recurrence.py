"""cp_recurrence, its gradient and its single step against the recurrence row by row in 64 bits."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from policy_util import TYPES, half_step, near, recurrence, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(rows, width, kind, *, seed=0, bias=True, h0=True, seqs=1, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[kind]
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(f=(rand(rows, width) * spread).to(dt).to(DEV), x=rand(rows, width).to(dt).to(DEV), dh=rand(rows, width).to(dt).to(DEV),
                bias=torch.linspace(0, 4, width).to(DEV) if bias else None, h0=rand(seqs, width).to(DEV) if h0 else None,
                dlast=rand(seqs, width).to(DEV))


def compare(d, ptr, reverse, packed, kind, what, dlast=True, **more):
    kw = dict(bias=d["bias"], h0=d["h0"], reverse=reverse)
    seq = torch.tensor(ptr, dtype=torch.int32, device=DEV) if packed else None
    dl = d["dlast"] if dlast else None
    ref, tol = recurrence(d["f"], d["x"], ptr, dh=d["dh"], dlast=dl, **kw)
    fwd = cpe.cp_recurrence(d["f"], d["x"], seq_ptr=seq, want_last=True, want_carry=True, **kw, **more)
    bwd = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], fwd["carry"], seq_ptr=seq, dlast=dl, **kw)
    got = {"h": fwd["h"], "last": fwd["last"], "df": bwd["df"], "dx": bwd["dx"]}
    if d["bias"] is not None:
        got["dbias"] = bwd["dbias"]
    if d["h0"] is not None:
        got["dh0"] = bwd["dh0"]
    for key, t in got.items():
        near(t, ref[key], tol[key] + half_step(t.dtype, ref[key]), f"{what} {key}")
    return fwd, bwd


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (2, 64), (15, 33), (17, 130), (127, 64), (128, 128), (129, 257), (500, 96), (1031, 66)])
def test_one_sequence(rows, width, kind):
    for reverse in (False, True):
        compare(make(rows, width, kind, seed=rows), [0, rows], reverse, False, kind, f"{rows}x{width} {kind} {reverse}")


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("ptr", [
    [0, 0], [0, 0, 0, 5], [0, 1, 2, 3, 4], [0, 16, 32, 48, 128, 256], [0, 128, 129, 129, 400], [0, 127, 128, 300, 300],
    [0, 5, 5, 5, 5, 140, 141, 142, 260, 260], [0] + [200] * 90 + [201, 333],
])
def test_packed_sequences(ptr, reverse):
    d = make(ptr[-1], 70, "fp32", seqs=len(ptr) - 1, seed=len(ptr))
    compare(d, ptr, reverse, True, "fp32", f"{ptr[:9]} {reverse}")


@pytest.mark.parametrize("reverse", [False, True])
def test_many_short_sequences(reverse):
    rng = np.random.default_rng(5)
    ptr = [0] + np.cumsum(rng.integers(0, 9, 700)).tolist()
    d = make(ptr[-1], 64, "bf16", seqs=700, seed=9)
    compare(d, ptr, reverse, True, "bf16", "700 sequences")


@pytest.mark.parametrize("bias,h0,dlast", [(False, False, False), (True, False, True), (False, True, False)])
def test_options(bias, h0, dlast):
    d = make(300, 40, "fp32", bias=bias, h0=h0, seqs=1)
    compare(d, [0, 300], False, False, "fp32", f"{bias} {h0} {dlast}", dlast=dlast)


def test_batches_are_sequences_of_equal_length():
    d = make(4 * 150, 48, "bf16", seqs=4)
    ptr = [0, 150, 300, 450, 600]
    flat, _ = compare(d, ptr, True, True, "bf16", "packed")
    cube = cpe.cp_recurrence(d["f"].view(4, 150, 48), d["x"].view(4, 150, 48), bias=d["bias"], h0=d["h0"], reverse=True, want_last=True)
    assert torch.equal(cube["h"].view(600, 48), flat["h"]) and torch.equal(cube["last"], flat["last"])


def test_strided_rows_and_outputs():
    # slices of one projection in, slices of one gradient out; an odd distance and an odd start too
    for wide_, lo in ((256, 0), (256, 64), (201, 1)):
        d = make(333, 64, "bf16", h0=False)
        buf = torch.zeros(333, wide_, dtype=torch.bfloat16, device=DEV)
        buf[:, lo:lo + 64], buf[:, lo + 64:lo + 128] = d["f"], d["x"]
        f, x = buf[:, lo:lo + 64], buf[:, lo + 64:lo + 128]
        plain = cpe.cp_recurrence(d["f"], d["x"], bias=d["bias"], want_carry=True)
        hbuf = torch.full_like(buf, 7.0)
        got = cpe.cp_recurrence(f, x, bias=d["bias"], want_carry=True, out={"h": hbuf[:, lo:lo + 64]})
        assert torch.equal(got["h"], plain["h"]) and (hbuf[:, lo + 64:] == 7).all() and (hbuf[:, :lo] == 7).all()
        grad = torch.full_like(buf, 7.0)
        a = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], plain["carry"], bias=d["bias"])
        b = cpe.cp_recurrence_backward(d["dh"], f, x, got["carry"], bias=d["bias"],
                                       out={"df": grad[:, lo:lo + 64], "dx": grad[:, lo + 64:lo + 128]})
        assert torch.equal(a["df"], b["df"]) and torch.equal(a["dx"], b["dx"]) and torch.equal(a["dbias"], b["dbias"])
        assert (grad[:, lo + 128:] == 7).all() and (grad[:, :lo] == 7).all()


def test_what_a_sequence_holds_stays_in_it():
    ptr = [0, 100, 300, 420]
    seq = torch.tensor(ptr, dtype=torch.int32, device=DEV)
    d = make(420, 64, "fp32", seqs=3)
    for reverse in (False, True):
        kw = dict(seq_ptr=seq, bias=d["bias"], h0=d["h0"], reverse=reverse, want_last=True, want_carry=True)
        want = cpe.cp_recurrence(d["f"], d["x"], **kw)
        x = d["x"].clone()
        x[150] = float("nan")
        x[40, :3] = float("inf")
        got = cpe.cp_recurrence(d["f"], x, **kw)
        assert torch.equal(got["h"][300:], want["h"][300:]) and torch.equal(got["last"][2], want["last"][2])
        assert got["h"][150].isnan().all()
        dh = d["dh"].clone()
        dh[150] = float("nan")
        back = dict(seq_ptr=seq, bias=d["bias"], h0=d["h0"], dlast=d["dlast"], reverse=reverse)
        a = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], want["carry"], **back)
        b = cpe.cp_recurrence_backward(dh, d["f"], d["x"], want["carry"], **back)
        for key in ("df", "dx"):
            assert torch.equal(a[key][:100], b[key][:100]) and torch.equal(a[key][300:], b[key][300:]), key


def test_gates_at_their_ends():
    # a = 0, a = 1 and everything between, where e^f is inf or 0
    f = torch.tensor([-200.0, -90.0, -30.0, 0.0, 20.0, 90.0, 200.0, float("-inf"), float("inf")]).repeat(300, 1).to(DEV)
    x = torch.randn(300, 9, generator=torch.Generator().manual_seed(3)).to(DEV)
    h0 = torch.ones(1, 9, device=DEV)
    fwd = cpe.cp_recurrence(f, x, h0=h0, want_carry=True)
    assert fwd["h"].isfinite().all()
    assert torch.equal(fwd["h"][:, 0], x[:, 0]) and torch.equal(fwd["h"][:, 7], x[:, 7])
    assert (fwd["h"][:, 6] == 1).all() and (fwd["h"][:, 8] == 1).all()
    bwd = cpe.cp_recurrence_backward(torch.ones_like(x), f, x, fwd["carry"], h0=h0)
    assert all(bwd[k].isfinite().all() for k in ("df", "dx", "dh0"))
    assert (bwd["dx"][:, 0] == 1).all() and (bwd["df"][:, [0, 6, 7, 8]] == 0).all()


def test_gradient_against_differences():
    d = make(200, 5, "fp32", seqs=3, seed=4)
    ptr = [0, 60, 61, 200]
    seq = torch.tensor(ptr, dtype=torch.int32, device=DEV)
    kw = dict(bias=d["bias"], h0=d["h0"])
    fwd = cpe.cp_recurrence(d["f"], d["x"], seq_ptr=seq, want_carry=True, **kw)
    bwd = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], fwd["carry"], seq_ptr=seq, dlast=d["dlast"], **kw)
    base = dict(f=d["f"].double().cpu(), x=d["x"].double().cpu(), bias=d["bias"].double().cpu(), h0=d["h0"].double().cpu())

    def loss(v):
        out, _ = recurrence(v["f"], v["x"], ptr, bias=v["bias"], h0=v["h0"])
        return (out["h"] * wide(d["dh"])).sum() + (out["last"] * wide(d["dlast"])).sum()

    g = torch.Generator().manual_seed(11)
    for key in base:
        way = torch.randn(base[key].shape, generator=g, dtype=torch.float64)
        step = 1e-5
        diff = (loss({**base, key: base[key] + step * way}) - loss({**base, key: base[key] - step * way})) / (2 * step)
        mine = (bwd["d" + key].double().cpu() * way).sum().item()
        # the difference's own error is step^2 times a third derivative, far below; the kernel's: U a term
        bound = 1e-6 * (bwd["d" + key].double().cpu() * way).abs().sum().item() + 1e-6
        assert abs(diff - mine) <= bound, (key, diff, mine)


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("count,width", [(1, 1), (3, 67), (8, 512), (300, 100)])
def test_step(count, width, kind):
    d = make(count, width, kind, seed=count, h0=False)
    g = torch.Generator().manual_seed(1)
    state = torch.randn(count + 3, width, generator=g).to(DEV)
    slots = torch.randperm(count + 3, generator=g)[:count].to(torch.int32)
    slots[count // 2] = -1 if count > 2 else slots[count // 2]
    for sl in (None, slots):
        st = state.clone()
        rows = list(range(count)) if sl is None else sl.tolist()
        got = cpe.cp_recurrence_step(d["f"], d["x"], st, bias=d["bias"], slots=None if sl is None else sl.to(DEV))
        want = wide(state)
        for i, row in enumerate(rows):
            if row < 0:
                assert (got["h"][i] == 0).all()
                continue
            ref, tol = recurrence(d["f"][i:i + 1], d["x"][i:i + 1], [0, 1], bias=d["bias"], h0=state[row:row + 1])
            near(got["h"][i:i + 1], ref["h"], tol["h"] + half_step(TYPES[kind], ref["h"]), f"row {i}")
            near(st[row], ref["h"][0], tol["h"][0] + half_step(torch.float32, ref["h"][0]), f"state {row}")
            want[row] = np.nan
        still = np.isfinite(want)
        assert np.array_equal(wide(st)[still], want[still])


def test_steps_continue_a_scan():
    d = make(130, 64, "fp32", h0=False)
    whole = cpe.cp_recurrence(d["f"], d["x"], bias=d["bias"], want_last=True)
    state = cpe.cp_recurrence(d["f"][:120], d["x"][:120], bias=d["bias"], want_last=True)["last"]
    for t in range(120, 130):
        h = cpe.cp_recurrence_step(d["f"][t:t + 1], d["x"][t:t + 1], state, bias=d["bias"])["h"]
        near(h, wide(whole["h"][t:t + 1]), 1e-5, f"step {t}")
    near(state, wide(whole["last"]), 1e-5)


def test_bad_sequences_and_slots_are_told():
    d = make(300, 64, "fp32", h0=False)
    for ptr in ([0, 200, 100, 300], [1, 300], [0, 299], [0, -5, 300], [0, 400, 300], [300, 0]):
        with pytest.raises(ValueError):
            cpe.cp_recurrence(d["f"], d["x"], seq_ptr=torch.tensor(ptr, dtype=torch.int32, device=DEV), want_last=True)
    state = torch.zeros(4, 64, device=DEV)
    with pytest.raises(ValueError):
        cpe.cp_recurrence_step(d["f"][:2], d["x"][:2], state, slots=torch.tensor([1, 4], dtype=torch.int32, device=DEV))
    assert (state[[0, 2, 3]] == 0).all() and (state[1] != 0).any()


def test_on_another_stream_and_in_a_graph():
    d = make(700, 96, "bf16", h0=False)
    want = cpe.cp_recurrence(d["f"], d["x"], bias=d["bias"], want_carry=True)
    grad = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], want["carry"], bias=d["bias"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cpe.cp_recurrence(d["f"], d["x"], bias=d["bias"], stream=side)
    side.synchronize()
    assert torch.equal(got["h"], want["h"])
    f, x, dh = (d[k].clone() for k in ("f", "x", "dh"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = cpe.cp_recurrence(f, x, bias=d["bias"], want_carry=True)
        b = cpe.cp_recurrence_backward(dh, f, x, a["carry"], bias=d["bias"])
    for turn in range(4):
        f.copy_(d["f"] if turn % 2 == 0 else d["x"])
        x.copy_(d["x"] if turn % 2 == 0 else d["f"])
        graph.replay()
        torch.cuda.synchronize()
        e = cpe.cp_recurrence(f, x, bias=d["bias"], want_carry=True)
        eb = cpe.cp_recurrence_backward(dh, f, x, e["carry"], bias=d["bias"])
        assert torch.equal(a["h"], e["h"]) and torch.equal(b["df"], eb["df"]) and torch.equal(b["dbias"], eb["dbias"])
        if turn % 2 == 0:
            assert torch.equal(e["h"], want["h"]) and torch.equal(eb["dbias"], grad["dbias"])


@pytest.mark.parametrize("rows,width,kind,reverse", [(20011, 34, "bf16", False), (9999, 7, "fp32", True), (16384, 1, "fp16", False)])
def test_sequences_of_many_tiles(rows, width, kind, reverse):
    # (more tiles than a group of them has)
    cuts = [0, rows // 2 + 3, rows // 2 + 3, rows - 5, rows]
    compare(make(rows, width, kind, seqs=4), cuts, reverse, True, kind, f"{rows} x {width} {kind}, four sequences")
    compare(make(rows, width, kind, seed=1), [0, rows], reverse, False, kind, f"{rows} x {width} {kind}, one sequence")


def test_results_do_not_depend_on_the_order_of_workgroups():
    d = make(150000, 96, "fp32", h0=False)
    kw = dict(bias=d["bias"], want_carry=True, want_last=True)
    one = cpe.cp_recurrence(d["f"], d["x"], **kw)
    grad = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], one["carry"], bias=d["bias"])
    for _ in range(5):
        again = cpe.cp_recurrence(d["f"], d["x"], **kw)
        assert all(torch.equal(again[k], one[k]) for k in ("h", "last", "carry"))
        back = cpe.cp_recurrence_backward(d["dh"], d["f"], d["x"], again["carry"], bias=d["bias"])
        assert all(torch.equal(back[k], grad[k]) for k in ("df", "dx", "dbias"))


def test_a_long_chain():
    compare(make(500003, 3, "bf16", seqs=3), [0, 7, 300001, 500003], True, True, "bf16", "half a million rows")
