"""cp_token_sample at the borders of its ways: many equal logits, long rows, more rows than a grid's first dimension, graphs and
streams; and partitions drawn for cp_eval."""
import numpy as np
import pytest
import torch

import paper_1711_01912_amd as cpe
from paper_1711_01912_amd import policy
from test_gpu_token_sample import FILTERS, check, inputs
from workloads import make_workload

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MORE = FILTERS + [dict(top_k=700), dict(top_k=3000), dict(top_k=3000, top_p=0.7), dict(top_p=0.999), dict(top_p=1e-9), dict(top_p=0.5, min_p=0.001)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [3500, 9000, 40000])
def test_few_values_many_times(V, dtype):
    # lists do not have room for what is alike: it is found by the digits of the keys
    logits, u = inputs(5, V, 4, dtype, seed=V)
    logits[0] = 1.0
    logits[1] = torch.round(logits[1])
    logits[2] = torch.where(logits[2] > 0, 3.0, -3.0).to(logits.dtype)
    logits[3] = logits[3] * 1e-3
    logits[4] = logits[4] * 30
    for f in MORE:
        check(logits, u, **f)
        check(logits, u, scale=40.0, **f)


@pytest.mark.parametrize("dtype,V", [("fp32", 1300001), ("bf16", 1100003), ("fp16", 200000)])
def test_long_rows(dtype, V):
    logits, u = inputs(2, V, 3, dtype, seed=1)
    for f in (dict(), dict(top_p=0.9), dict(top_k=100, top_p=0.95), dict(top_k=20000), dict(min_p=0.01), dict(top_p=0.3, min_p=0.001)):
        check(logits, u, **f)


@pytest.mark.parametrize("V", [9000, 30000])
def test_more_rows_than_compute_units(V):
    logits, u = inputs(300, V, 1, "bf16", seed=V)
    for f in (dict(top_p=0.9), dict(top_k=30), dict(min_p=0.05)):
        check(logits, u, **f)


SLICED = [dict(top_k=1), dict(top_k=50, top_p=0.9), dict(top_k=50, min_p=0.01), dict(top_k=128), dict(top_k=129), dict(top_k=256), dict(top_p=0.0), dict(top_p=0.9), dict(min_p=0.2)]


@pytest.mark.parametrize("dtype,V", [("fp32", 65536), ("bf16", 80001), ("fp16", 70000), ("bf16", 524289)])
def test_few_long_rows(V, dtype):
    # what is kept lies in one slice, in the last, in all; what is alike has room in no list
    logits, u = inputs(9, V, 2, dtype, seed=V)
    logits[1] = 1.0
    logits[2] = -float("inf")
    logits[2, V - 3:] = 2.0
    logits[3] = -float("inf")
    logits[3, 8190:8194] = torch.tensor([1.0, 2.0, 2.0, 1.0])
    logits[4] = logits[4].sort().values
    logits[5] = torch.round(logits[5])
    logits[6, V // 2], logits[7, V - 1] = float("nan"), float("inf")
    logits[8] = -float("inf")
    for f in SLICED:
        check(logits, u, scale=0.7, **f)
    allowed = np.random.default_rng(V).random((9, V)) < 0.3
    allowed[6, V // 2] = allowed[7, V - 1] = False
    allowed[4, 100:] = False
    for f in SLICED[1:4]:
        check(logits, u, allowed, **f)


def test_few_long_rows_with_settings_of_their_own():
    logits, u = inputs(64, 66000, 3, "bf16", seed=4)
    g = np.random.default_rng(4)
    k, p = g.choice([0, 1, 3, 50, 127, 128, 129, 256, 1024, 1025, 66000, 70000], 64), g.choice([0.0, 0.3, 0.9, 1.0], 64)
    check(logits, u, top_k=k, top_p=p, min_p=g.choice([0.0, 0.01], 64))
    check(logits, u, top_p=p)
    k[5], p[6] = -1, 1.5
    out = cpe.cp_token_sample(logits.to(DEV), u.to(DEV), top_k=torch.tensor(k, dtype=torch.int32, device=DEV), top_p=torch.tensor(p, dtype=torch.float32, device=DEV),
                              check_status=False)
    assert int(out["status"]) == policy.STATUS_BAD_SAMPLING and bool((out["tokens"][5:7] == -1).all()) and int((out["tokens"] == -1).sum()) == 6
    # rows of one buffer at odd places, and a graph
    wide = torch.zeros(8, 66100, dtype=torch.bfloat16, device=DEV)
    wide[:, 7:66007] = logits[:8].to(DEV)
    u = u[:8].to(DEV)
    want = cpe.cp_token_sample(logits[:8].to(DEV), u, top_k=50, top_p=0.9)["tokens"]
    assert torch.equal(cpe.cp_token_sample(wide[:, 7:66007], u, top_k=50, top_p=0.9)["tokens"], want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cpe.cp_token_sample(wide[:, 7:66007], u, top_k=50, top_p=0.9)
    for turn in range(3):
        u.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(turn)))
        want = cpe.cp_token_sample(wide[:, 7:66007], u, top_k=50, top_p=0.9)["tokens"]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["tokens"], want)


def test_sorted_rows():
    logits, u = inputs(4, 20000, 5, "fp32", seed=2)
    logits[0], logits[1] = logits[0].sort().values, logits[1].sort(descending=True).values
    logits[2, :10000] = -float("inf")
    logits[3, 100:] = -float("inf")
    for f in MORE:
        check(logits, u, **f)


@pytest.mark.parametrize("V", [5, 257])
def test_more_rows_than_a_grid_s_first_dimension_has(V):
    rows = 2 ** 22 * (32 if V == 5 else 1) + 3          # (32 rows of 5 places a workgroup)
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.empty(rows, V, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    u = torch.rand(rows, generator=g, device=DEV)
    tok = cpe.cp_token_sample(x, u, top_k=3, dtype=torch.int32)["tokens"]
    for lo in (0, 2 ** 22 - 2, rows // 2, rows - 4):
        assert torch.equal(tok[lo:lo + 4], cpe.cp_token_sample(x[lo:lo + 4], u[lo:lo + 4], top_k=3, dtype=torch.int32)["tokens"]), lo
    assert int(tok.min()) >= 0 and int(tok.max()) < V


def test_rows_beyond_32_bits():
    buffer = torch.zeros(40 * 2 ** 26 + 1000, dtype=torch.bfloat16, device=DEV)
    x = torch.randn(40, 900, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    view = buffer.as_strided((40, 900), (2 ** 26, 1))
    view.copy_(x)
    u = torch.rand(40, 2, device=DEV)
    for cols in (900, 200, 7):
        assert torch.equal(cpe.cp_token_sample(view[:, :cols], u, top_p=0.9)["tokens"], cpe.cp_token_sample(x[:, :cols].contiguous(), u, top_p=0.9)["tokens"])


@pytest.mark.parametrize("V", [8, 100, 2000, 20000])
def test_calls_in_graphs_and_on_streams(V):
    logits, u = (t.to(DEV) for t in inputs(20, V, 3, "bf16", seed=V))
    rows = dict(top_k=torch.randint(0, 60, (20,), generator=torch.Generator().manual_seed(V)).to(torch.int32).to(DEV), top_p=torch.full((20,), 0.9, device=DEV))
    one = lambda **kw: cpe.cp_token_sample(logits, u, want_logp=True, check_status=False, **rows, **kw)  # noqa: E731
    want = one()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = one(stream=stream)
    stream.synchronize()
    assert torch.equal(got["tokens"], want["tokens"]) and torch.equal(got["logp"], want["logp"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one()
    for turn in range(3):
        u.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(turn)))
        want = one()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["tokens"], want["tokens"]) and torch.equal(out["logp"], want["logp"]) and int(out["status"]) == 0


def test_partitions_for_cp_eval(oracle):
    # drawn in either layout, rated by cp_eval, and their log probabilities those of cp_token_logprobs where nothing is left out
    w = make_workload("tiny")
    g = torch.Generator().manual_seed(1)
    logits, u = torch.randn(w.n, w.k, generator=g).to(DEV), torch.rand(w.n, 40, generator=g).to(DEV)
    got = cpe.cp_token_sample(logits, u, dtype=torch.uint8, want_logp=True)
    parts = torch.empty(40, w.n, dtype=torch.uint8, device=DEV)
    cpe.cp_token_sample(logits, u, out=dict(tokens=parts.t()))
    assert torch.equal(parts.t(), got["tokens"])
    logp = cpe.cp_token_logprobs(logits, got["tokens"])["logp"]
    # (32 bits there: the operator's own tolerance, some 200 steps of 2^-24 and 4 for each unit of the exponent)
    assert float((logp - got["logp"]).abs().max()) <= 2.0 ** -24 * (200 + 4 * 12)
    graph = cpe.CpGraph.from_workload(w, device=DEV)
    cp = cpe.cp_eval(graph, parts, w.speeds, w.bandwidth, want=("cp",))["cp"].cpu().numpy()
    ref = oracle.evaluate(w.n, w.succ_ptr, w.succ_idx, w.succ_t, w.c, w.speeds, w.bandwidth, parts.cpu().numpy())["cp"]
    assert np.array_equal(cp, ref)
