"""cp_norm_gate and its gradient against the formulas in 64 bits."""
import pytest
import torch

import paper_1711_01912_amd as cpe
from paper_1711_01912_amd import policy
from policy_util import TYPES, half_step, joint, near, wide

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(rows, width, block, stream, weights=None, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    tb, ts = TYPES[block], TYPES[stream]
    tw = TYPES[weights or block]
    return dict(x=(3 * spread * rand(rows, width)).to(ts).to(DEV), y=(2 * rand(rows, width)).to(tb).to(DEV), gate=rand(rows, width).to(tb).to(DEV),
                w_pre=(1 + 0.2 * rand(width)).to(tw).to(DEV), w_post=(1 + 0.2 * rand(width)).to(tw).to(DEV),
                dr=rand(rows, width).to(ts).to(DEV), dz=rand(rows, width).to(tb).to(DEV))


def compare(d, what, *, gate=True, post=True, act="sigmoid", scale=0.5, eps=1e-6, dr=True, y=True):
    yy, gt = d["y"] if y else None, d["gate"] if gate and y else None
    post_ = d["w_post"] if post and y else None
    drr = d["dr"] if dr else None
    kw = dict(w_pre=d["w_pre"], w_post=post_, gate_act=act, scale=scale)
    ref, tol = joint(d["x"], yy, gt, d["w_pre"], post_, act, scale, eps, dr=drr, dz=d["dz"])
    fwd = cpe.cp_norm_gate(d["x"], yy, gt, eps=eps, want_stats=True, z_dtype=d["dz"].dtype, **kw)
    bwd = cpe.cp_norm_gate_backward(drr, d["dz"], d["x"], yy, gt, stats=fwd["stats"], **kw)
    got = {"z": fwd["z"], "dx": bwd["dx"], "dw_pre": bwd["dw_pre"]}
    if y:
        got.update(r=fwd["r"], dy=bwd["dy"])
    if gt is not None:
        got["dgate"] = bwd["dgate"]
    if post_ is not None:
        got["dw_post"] = bwd["dw_post"]
    assert set(got) == {k for k in ref if k != "r" or y}
    for key, t in got.items():
        near(t, ref[key], tol[key] + half_step(t.dtype, ref[key]), f"{what} {key}")
    return fwd, bwd


@pytest.mark.parametrize("block,stream", [("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32")])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (2, 63), (5, 64), (4, 257), (130, 512), (7, 1111), (3, 2048), (2, 4100)])
def test_sizes_and_types(rows, width, block, stream):
    compare(make(rows, width, block, stream, seed=width), f"{rows}x{width} {block} {stream}")


@pytest.mark.parametrize("width", [8191, 8192, 16383, 16384])
def test_widest_rows(width):
    compare(make(3, width, "bf16", "bf16", seed=2), f"{width}")


@pytest.mark.parametrize("act", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("gate,post,dr,y", [(True, True, True, True), (True, False, False, True), (False, True, True, True),
                                            (False, False, True, True), (False, False, True, False), (False, False, False, False)])
def test_options(act, gate, post, dr, y):
    compare(make(33, 96, "bf16", "fp32", weights="fp32", seed=1), f"{act} {gate} {post} {dr} {y}", gate=gate, post=post, act=act, dr=dr, y=y)


def test_many_rows_for_the_weights():
    compare(make(5000, 72, "bf16", "bf16", weights="fp32", seed=3), "5000 rows")


def test_rows_of_zeros_and_large_gates():
    d = make(6, 128, "fp32", "fp32", seed=4)
    d["y"][1] = 0
    d["x"][2] = 0
    d["y"][2] = 0
    d["gate"][3] = 300.0
    d["gate"][4] = -300.0
    for act in ("sigmoid", "silu"):
        compare(d, act, act=act)
    got = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], w_pre=d["w_pre"], w_post=d["w_post"])
    assert (got["z"][2] == 0).all() and got["z"].isfinite().all()


def test_a_bad_row_stays_alone():
    d = make(40, 256, "bf16", "bf16")
    kw = dict(w_pre=d["w_pre"], w_post=d["w_post"])
    want = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], **kw)
    y = d["y"].clone()
    y[17, 5] = float("nan")
    got = cpe.cp_norm_gate(d["x"], y, d["gate"], **kw)
    keep = [i for i in range(40) if i != 17]
    assert torch.equal(got["z"][keep], want["z"][keep]) and torch.equal(got["r"][keep], want["r"][keep])
    assert got["z"][17].isnan().all()


def test_strided_rows():
    for wide_, lo in ((512, 128), (301, 3)):
        d = make(50, 96, "bf16", "bf16")
        kw = dict(w_pre=d["w_pre"], w_post=d["w_post"])
        fwd = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], want_stats=True, **kw)
        bwd = cpe.cp_norm_gate_backward(d["dr"], d["dz"], d["x"], d["y"], d["gate"], stats=fwd["stats"], **kw)
        v = {}
        for key in ("x", "y", "gate", "dr", "dz"):
            buf = torch.zeros(50, wide_, dtype=torch.bfloat16, device=DEV)
            v[key] = buf[:, lo:lo + 96]
            v[key].copy_(d[key])
        outs = {k: torch.full((50, wide_), 5.0, dtype=torch.bfloat16, device=DEV) for k in ("r", "z", "dx", "dy", "dgate")}
        cut = {k: t[:, lo:lo + 96] for k, t in outs.items()}
        f2 = cpe.cp_norm_gate(v["x"], v["y"], v["gate"], want_stats=True, out={"r": cut["r"], "z": cut["z"]}, **kw)
        b2 = cpe.cp_norm_gate_backward(v["dr"], v["dz"], v["x"], v["y"], v["gate"], stats=f2["stats"],
                                       out={k: cut[k] for k in ("dx", "dy", "dgate")}, **kw)
        for key in ("r", "z"):
            near(f2[key], wide(fwd[key]), half_step(torch.bfloat16, wide(fwd[key])) * 2, key)
        for key in ("dx", "dy", "dgate", "dw_pre", "dw_post"):
            near(b2[key], wide(bwd[key]), half_step(torch.bfloat16, wide(bwd[key])) * 2 + 1e-6, key)
        assert all((t[:, :lo] == 5).all() and (t[:, lo + 96:] == 5).all() for t in outs.values())


def test_gradient_against_differences():
    d = make(9, 20, "fp32", "fp32", seed=6)
    kw = dict(w_pre=d["w_pre"], w_post=d["w_post"], gate_act="silu", scale=0.7)
    fwd = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], want_stats=True, **kw)
    bwd = cpe.cp_norm_gate_backward(d["dr"], d["dz"], d["x"], d["y"], d["gate"], stats=fwd["stats"], **kw)
    names = ("x", "y", "gate", "w_pre", "w_post")
    base = {k: d[k].double().cpu() for k in names}

    def loss(v):
        out, _ = joint(v["x"], v["y"], v["gate"], v["w_pre"], v["w_post"], "silu", 0.7, 1e-6)
        return (out["r"] * wide(d["dr"])).sum() + (out["z"] * wide(d["dz"])).sum()

    g = torch.Generator().manual_seed(2)
    for key in names:
        way = torch.randn(base[key].shape, generator=g, dtype=torch.float64)
        diff = (loss({**base, key: base[key] + 1e-5 * way}) - loss({**base, key: base[key] - 1e-5 * way})) / 2e-5
        terms = bwd["d" + key].double().cpu() * way
        assert abs(diff - terms.sum().item()) <= 2e-6 * terms.abs().sum().item() + 1e-6, key


def test_no_rows():
    d = make(4, 64, "bf16", "bf16")
    e = {k: d[k][:0] for k in ("x", "y", "gate", "dr", "dz")}
    kw = dict(w_pre=d["w_pre"], w_post=d["w_post"])
    fwd = cpe.cp_norm_gate(e["x"], e["y"], e["gate"], want_stats=True, **kw)
    assert fwd["z"].shape == (0, 64)
    bwd = cpe.cp_norm_gate_backward(e["dr"], e["dz"], e["x"], e["y"], e["gate"], stats=fwd["stats"], **kw)
    assert (bwd["dw_pre"] == 0).all() and (bwd["dw_post"] == 0).all()


def test_in_a_graph():
    d = make(300, 256, "bf16", "bf16")
    kw = dict(w_pre=d["w_pre"], w_post=d["w_post"])
    x = d["x"].clone()
    cpe.cp_norm_gate(x, d["y"], d["gate"], **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = cpe.cp_norm_gate(x, d["y"], d["gate"], want_stats=True, **kw)
        b = cpe.cp_norm_gate_backward(d["dr"], d["dz"], x, d["y"], d["gate"], stats=a["stats"], **kw)
    for turn in range(3):
        x.copy_(d["x"] * (1 + turn))
        graph.replay()
        torch.cuda.synchronize()
        e = cpe.cp_norm_gate(x, d["y"], d["gate"], want_stats=True, **kw)
        eb = cpe.cp_norm_gate_backward(d["dr"], d["dz"], x, d["y"], d["gate"], stats=e["stats"], **kw)
        assert torch.equal(a["z"], e["z"]) and torch.equal(b["dx"], eb["dx"]) and torch.equal(b["dw_pre"], eb["dw_pre"])


@pytest.mark.parametrize("block,stream", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,width", [(9, 3), (1001, 7), (517, 31), (77, 65), (131, 127), (40000, 33)])
def test_rows_side_by_side(rows, width, block, stream):
    compare(make(rows, width, block, stream, weights="fp32", seed=width), f"{rows}x{width} {block} {stream}")


@pytest.mark.parametrize("width", [5, 64, 72, 200, 1000])
def test_the_workspace_is_as_large_as_said(width):
    for block, stream in (("bf16", "bf16"), ("bf16", "fp32")):
        d = make(70000, width, block, stream, weights="fp32")
        kw = dict(w_pre=d["w_pre"], w_post=d["w_post"])
        fwd = cpe.cp_norm_gate(d["x"], d["y"], d["gate"], want_stats=True, **kw)
        need = policy._need("cp_norm_gate_backward_workspace_bytes", 70000, width)
        room = torch.full((need + 4096,), 7, dtype=torch.uint8, device=DEV)
        one = cpe.cp_norm_gate_backward(None, d["dz"], d["x"], d["y"], d["gate"], stats=fwd["stats"], workspace=room[:need], **kw)
        assert (room[need:] == 7).all()
        two = cpe.cp_norm_gate_backward(None, d["dz"], d["x"], d["y"], d["gate"], stats=fwd["stats"], **kw)
        assert torch.equal(one["dw_pre"], two["dw_pre"]) and torch.equal(one["dw_post"], two["dw_post"])
