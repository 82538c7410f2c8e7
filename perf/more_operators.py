"""More operators of a learned placement policy, as measurable cases.

Next to the gated recurrence a policy's sequence layer may keep a matrix a head as its state: linear
attention with a decay for each head (cp_linear_attention with its gradient, over whole sequences;
cp_linear_attention_step, one more vertex or token of many sequences).  At the other end the policy's
rows of logits become partitions or tokens: cp_token_sample draws them from given random numbers,
with temperature, top-k, top-p and min-p.

    S_t = exp(log_decay_h) S_{t-1} + k_t^T v_t,      o_t = scale q_t S_t
    token = the first kept place whose cumulated probability exceeds u

``own`` false: elementary torch operations, in 32 bits for the attention (64 in the decays' gradient, a
long sum) and in 64 bits for the draws, where random numbers lie next to borders.  ``own`` true: the
package's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
TOKENS = {"uint8": torch.uint8, "int32": torch.int32, "int64": torch.int64}
TOKEN_SIZE = {"uint8": 1, "int32": 4, "int64": 8}


def listed():
    return [
        # eight graphs whose vertices are placed one by one: latency of one step
        dict(name="step-8", op="step", S=8, H=8, KV=8, K=64, V=64, dtype="bf16", slots=False),
        # a full house of sequences, their states kept in slots of a larger pool
        dict(name="step-512-slots", op="step", S=512, H=16, KV=16, K=128, V=128, dtype="bf16", slots=True),
        # odd widths, four heads on one of keys and values
        dict(name="step-odd-shared", op="step", S=133, H=12, KV=3, K=72, V=104, dtype="fp32", slots=True),
        # eight layers of eight vertices: launches and host time
        dict(name="attend-tiny", op="attend", S=1, N=64, H=4, KV=4, K=32, V=32, ragged=False, dtype="fp32", h0=False,
             reverse=False, train=False),
        # one long prompt read once, its last state kept for the steps that follow
        dict(name="attend-long", op="attend", S=1, N=65536, H=16, KV=16, K=128, V=128, ragged=False, dtype="bf16",
             h0=False, reverse=False, train=False),
        # a training batch of equally long sequences
        dict(name="attend-train-batch", op="attend", S=8, N=32768, H=16, KV=16, K=128, V=128, ragged=False, dtype="bf16",
             h0=False, reverse=False, train=True),
        # graphs of all sizes packed one behind the other, read from the sinks back, odd widths, shared keys and values
        dict(name="attend-train-ragged", op="attend", S=37, N=52710, H=6, KV=3, K=48, V=80, ragged=True, dtype="fp16",
             h0=True, reverse=True, train=True),
        # the benchmark's graph: a million vertices as one sequence, forward and backward
        dict(name="attend-train-million", op="attend", S=1, N=1000000, H=4, KV=4, K=64, V=64, ragged=False, dtype="bf16",
             h0=False, reverse=False, train=True),
        # single tokens of eight sequences over a large vocabulary
        dict(name="sample-8", op="sample", R=8, V=131072, G=1, dtype="bf16", tokens="int64", allow=False,
             scale=1.25, top_k=50, top_p=0.9, min_p=0.0, rows=False, logp=True),
        # a full batch whose sequences each have settings of their own
        dict(name="sample-512-rows", op="sample", R=512, V=65536, G=1, dtype="bf16", tokens="int32", allow=False,
             scale=1.0, top_k=200, top_p=0.95, min_p=0.02, rows=True, logp=True),
        # the paper's largest graph on fifty devices, some of which a vertex may not use; unlikely devices are left out
        dict(name="sample-devices", op="sample", R=5271, V=50, G=333, dtype="fp32", tokens="int32", allow=True,
             scale=0.8, top_k=0, top_p=0.95, min_p=0.01, rows=False, logp=True),
        # a thousand partitions of a wide graph over eight devices
        dict(name="sample-partitions", op="sample", R=200000, V=8, G=1024, dtype="bf16", tokens="uint8", allow=False,
             scale=1.0, top_k=0, top_p=1.0, min_p=0.0, rows=False, logp=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "attend", "attend", "attend", "vocabulary", "vocabulary", "devices"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind in ("step", "attend"):
        H = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
        KV = H if rng.random() < 0.7 else rng.choice([d for d in (1, 2, 3, 4) if H % d == 0])
        K, V = _log(rng, 16, 256), _log(rng, 16, 256)
        if rng.random() < 0.5:
            K = V = rng.choice([32, 64, 128])
        if kind == "step":
            S = _log(rng, 1, max(1, min(4096, 134217728 // (H * K * V))))
            return dict(op="step", S=S, H=H, KV=KV, K=K, V=V, dtype=dtype, slots=rng.random() < 0.5)
        N = _log(rng, 1, min(200000, 200000000 // (H * (K + V)), 4000000000 // (H * K * V)))
        ragged = N > 200 and rng.random() < 0.5
        S = _log(rng, 2, 64) if ragged else rng.choice([1, 1, 4, 16])
        S = S if ragged or N >= S else 1
        return dict(op="attend", S=S, N=N if ragged else N // S * S, H=H, KV=KV, K=K, V=V, ragged=ragged, dtype=dtype,
                    h0=rng.random() < 0.5, reverse=rng.random() < 0.3, train=rng.random() < 0.5)
    case = dict(op="sample", scale=rng.choice([0.7, 1.0, 1.4]), top_k=rng.choice([0, 0, 1, 40, 1000]),
                top_p=rng.choice([1.0, 0.9, 0.5]), min_p=rng.choice([0.0, 0.0, 0.05]), rows=rng.random() < 0.3,
                dtype=dtype, allow=rng.random() < 0.3, logp=rng.random() < 0.6)
    if kind == "vocabulary":
        V = _log(rng, 300, 200000)
        return dict(case, R=_log(rng, 1, 33554432 // V), V=V, G=rng.choice([1, 1, 4]), tokens=rng.choice(["int32", "int64"]))
    G = _log(rng, 1, 1024)
    return dict(case, R=_log(rng, 64, min(1000000, 200000000 // G)), V=_log(rng, 2, 64), G=G,
                tokens=rng.choice(["uint8", "int32"]))


# ---- inputs --------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    dt = TYPES[case["dtype"]]

    def normal(*shape, to=dt, by=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(by).to(to)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE)

    s = dict(case=dict(case))
    if case["op"] == "sample":
        R, V, G = case["R"], case["V"], case["G"]
        s["logits"] = normal(R, V, by=2.5)
        s["u"] = uniform(R, G)
        s["allow"] = None
        if case["allow"]:
            # a mask per row that forbids a third, some rows all: 64 places a word
            mask = uniform(R, -(-V // 64) * 64) < 0.67
            mask[:, V:] = False
            mask[uniform(R) < 0.02] = False
            bits = torch.ones(64, dtype=torch.int64, device=DEVICE) << torch.arange(64, device=DEVICE)
            s["allow"] = torch.stack([(mask[:, w * 64:w * 64 + 64] * bits).sum(-1) for w in range(-(-V // 64))], 1)
        s.update(scale=case["scale"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
        if case["rows"]:
            # requests with settings of their own: some take all there is, some only the best
            s["scale"] = 0.5 + 1.5 * uniform(R)
            s["top_k"] = torch.where(uniform(R) < 0.4, 0, (1 + uniform(R) * 2 * max(case["top_k"], 1)).floor()).to(torch.int32)
            s["top_p"] = torch.where(uniform(R) < 0.3, 1.0, 0.3 + 0.69 * uniform(R))
            s["min_p"] = torch.where(uniform(R) < 0.5, 0.0, 0.1 * uniform(R))
        return s
    S, H, KV, K, V = (case[n] for n in ("S", "H", "KV", "K", "V"))
    # from heads that look two positions back to such as look back thousands
    s["log_decay"] = -torch.exp(math.log(2e-4) + (math.log(0.7) - math.log(2e-4)) * uniform(H))
    s["scale"] = K ** -0.5
    N = S if case["op"] == "step" else case["N"]
    s["q"], s["k"], s["v"] = normal(N, H, K), normal(N, KV, K), normal(N, KV, V)
    if case["op"] == "step":
        pool = S + S // 4 + 1 if case["slots"] else S
        s["state"] = normal(pool, H, K, V, to=torch.float32)
        s["slots"] = None
        if case["slots"]:
            slots = torch.randperm(pool, generator=g, device=DEVICE)[:S].to(torch.int32)
            slots[S // 3:S // 3 + S // 50] = -1        # sequences that ended
            s["slots"] = slots
        return s
    s["seq_ptr"] = None
    if case["ragged"]:
        cuts = torch.randint(0, N + 1, (S - 1,), generator=g, device=DEVICE).sort().values
        if S > 4:
            cuts[1] = cuts[0]                          # a graph without vertices, and one of a single vertex
            cuts[3] = torch.minimum(cuts[2] + 1, cuts[3])
        ends = torch.tensor([0, N], device=DEVICE)
        s["seq_ptr"] = torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)
    s["h0"] = normal(S, H, K, V, to=torch.float32) if case["h0"] else None
    if case["train"]:
        s["do"] = normal(N, H, V)
        s["dlast"] = normal(S, H, K, V, to=torch.float32) if case["h0"] else None
    return s


# ---- one pass ------------------------------------------------------------------------------------


def run(s):
    return {"step": _step, "attend": _attend, "sample": _sample}[s["case"]["op"]](s)


def _step(s):
    if own:
        import paper_1711_01912_amd as cpe
        o = cpe.cp_linear_attention_step(s["q"], s["k"], s["v"], s["state"], s["log_decay"], scale=s["scale"], slots=s["slots"],
                                         check_status=False)["o"]
        return {"o": o, "state": s["state"]}
    state, slots, H = s["state"], s["slots"], s["case"]["H"]
    q, k, v = s["q"].float(), _per_head(s["k"].float(), H), _per_head(s["v"].float(), H)
    at = torch.arange(q.shape[0], device=DEVICE) if slots is None else slots.long()
    live = (at >= 0).view(-1, 1, 1)
    at = at.clamp(min=0)
    old = state[at]
    new = torch.exp(s["log_decay"]).view(-1, 1, 1) * old + k.unsqueeze(-1) * v.unsqueeze(-2)
    o = s["scale"] * (q.unsqueeze(-1) * new).sum(-2)
    if slots is None:
        state.copy_(new)
    else:
        # (sequences without a slot write to a row behind the last)
        spare = torch.cat([state, state[:1]])
        spare[torch.where(live.view(-1), at, state.shape[0])] = new
        state.copy_(spare[:-1])
    return {"o": torch.where(live, o, 0.0).to(s["q"].dtype), "state": state}


def _per_head(t, H):
    """[rows][kv heads][..] as [rows][heads][..]: neighbouring heads share."""
    return t if t.shape[1] == H else t.repeat_interleave(H // t.shape[1], 1)


def _doubling(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, in log2(N) rounds of products and sums."""
    n, k = a.shape[0], 1
    while k < n:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


CHUNK = 128


def _attend(s):
    case = s["case"]
    N, S, H, KV, K, V = (case[n] for n in ("N", "S", "H", "KV", "K", "V"))
    if own:
        import paper_1711_01912_amd as cpe
        lead = (N,) if case["ragged"] else (S, N // S)
        q, k, v = s["q"].view(*lead, H, K), s["k"].view(*lead, KV, K), s["v"].view(*lead, KV, V)
        kw = dict(scale=s["scale"], seq_ptr=s["seq_ptr"], h0=s["h0"], reverse=case["reverse"], check_status=False)
        fwd = cpe.cp_linear_attention(q, k, v, s["log_decay"], want_last=True, want_carry=case["train"], **kw)
        out = {"o": fwd["o"].view(N, H, V), "last": fwd["last"]}
        if case["train"]:
            bwd = cpe.cp_linear_attention_backward(s["do"].view(*lead, H, V), q, k, v, s["log_decay"], fwd["carry"],
                                                   dlast=s["dlast"], **kw)
            out.update(dq=bwd["dq"].view(N, H, K), dk=bwd["dk"].view(N, KV, K), dv=bwd["dv"].view(N, KV, V),
                       dlog_decay=bwd["dlog_decay"])
            if s["h0"] is not None:
                out["dh0"] = bwd["dh0"]
        return out
    turn = (lambda t: t.flip(0)) if case["reverse"] else (lambda t: t)
    dt, scale, g = s["q"].dtype, s["scale"], s["log_decay"]
    ptr = s["seq_ptr"].long() if s["seq_ptr"] is not None else torch.arange(S + 1, device=DEVICE) * (N // S)
    if case["reverse"]:
        ptr = N - ptr.flip(0)
    h0 = turn(s["h0"]) if s["h0"] is not None else torch.zeros(S, H, K, V, device=DEVICE)
    # chunks of CHUNK rows that begin anew with each sequence; those behind the last one hold no rows
    C, M = CHUNK, N // CHUNK + S
    chunks = (ptr[1:] - ptr[:-1] + C - 1) // C
    upto = chunks.cumsum(0)
    c = torch.arange(M, device=DEVICE)
    seq = torch.searchsorted(upto, c, right=True)
    there = seq < S
    seq = seq.clamp(max=S - 1)
    part = c - (upto - chunks)[seq]
    start = ptr[seq] + part * C
    count = torch.where(there, (ptr[seq + 1] - start).clamp(max=C), 0)
    first, final = there & (part == 0), there & (part == chunks[seq] - 1)
    inside = torch.arange(C, device=DEVICE) < count.unsqueeze(1)
    row = (start.unsqueeze(1) + torch.arange(C, device=DEVICE)).clamp(max=max(N - 1, 0))

    def cut(t):
        """[chunks][heads][C][width] of rows, zeros where a chunk has none"""
        t = _per_head(turn(t).float(), H)[row]
        return torch.where(inside.view(M, C, 1, 1), t, 0.0).permute(0, 2, 1, 3).contiguous()

    def join(t):
        out = torch.zeros(N + 1, H, t.shape[-1], device=DEVICE)
        out[torch.where(inside, row, N)] = t.permute(0, 2, 1, 3)
        return turn(out[:N])

    def shared(t):
        return t.view(N, KV, H // KV, -1).sum(2)

    q, k, v = cut(s["q"]), cut(s["k"]), cut(s["v"])
    pos = torch.arange(C, device=DEVICE, dtype=torch.float32)
    apart = pos.view(-1, 1) - pos
    within = torch.where(apart >= 0, torch.exp(g.view(-1, 1, 1) * apart.clamp(min=0)), 0.0)     # [H][C][C]
    entering = torch.exp(g.view(-1, 1) * (pos + 1)).view(1, H, C, 1)
    behind = (count.view(-1, 1) - 1 - pos).clamp(min=0)                                         # rows from j to a chunk's end
    leaving = torch.exp(g.view(1, H, 1) * behind.view(M, 1, C)).unsqueeze(-1)
    through = torch.exp(g.view(1, -1) * count.view(-1, 1)).view(M, H, 1, 1)
    firsts = first.view(M, 1, 1, 1)
    added = (k * leaving).transpose(2, 3).contiguous() @ v
    added = added + torch.where(firsts, through * h0[seq], 0.0)
    after = _doubling(torch.where(firsts, 0.0, through), added)                                 # the state behind each chunk
    before = torch.where(firsts, h0[seq], torch.cat([after[:1], after[:-1]]))
    scores = q @ k.transpose(2, 3).contiguous()
    passed = q @ before
    o = scale * ((scores * within) @ v + entering * passed)
    last = h0.clone()
    where = torch.where(final, seq, S)
    last = torch.cat([last, last[:1]])
    last[where] = after
    out = {"o": join(o).to(dt), "last": turn(last[:S])}
    if not case["train"]:
        return out
    do = cut(s["do"])
    dlast = turn(s["dlast"]) if s["dlast"] is not None else torch.zeros(S, H, K, V, device=DEVICE)
    # gradient of the state behind each chunk, from the last chunk on
    finals = final.view(M, 1, 1, 1)
    enters = scale * ((q * entering).transpose(2, 3).contiguous() @ do)        # of the state before, by the chunk's own rows
    step = torch.where(finals, through * dlast[seq], 0.0) + enters
    gain = torch.where(finals, 0.0, through)
    dbefore = _doubling(gain.flip(0), step.flip(0)).flip(0)
    dafter = torch.where(finals, dlast[seq], torch.cat([dbefore[1:], dbefore[:1]]))
    dscores = do @ v.transpose(2, 3).contiguous()
    dp = dscores * within
    back = do @ before.transpose(2, 3).contiguous()
    dq = scale * (dp @ k + entering * back)
    kd = leaving * (v @ dafter.transpose(2, 3).contiguous())
    dk = scale * (dp.transpose(2, 3).contiguous() @ q) + kd
    dv = scale * ((scores * within).transpose(2, 3).contiguous() @ do) + leaving * (k @ dafter)
    decay = (scale * apart.clamp(min=0) * scores * dp).sum((2, 3))
    decay = decay + scale * ((pos + 1).view(1, 1, C) * (entering * passed * do).sum(-1)).sum(-1)
    decay = decay + (behind.view(M, 1, C) * (k * kd).sum(-1)).sum(-1)
    decay = decay + count.view(M, 1) * (through * before * dafter).sum((2, 3))
    out.update(dq=join(dq).to(dt), dk=shared(join(dk)).to(dt), dv=shared(join(dv)).to(dt),
               dlog_decay=decay.sum(0, dtype=torch.float64).float())
    if s["h0"] is not None:
        dh0 = torch.cat([dlast, dlast[:1]])
        dh0[torch.where(first, seq, S)] = dbefore
        out["dh0"] = turn(dh0[:S])
    return out


def _sample(s):
    case = s["case"]
    V = case["V"]
    if own:
        import paper_1711_01912_amd as cpe
        got = cpe.cp_token_sample(s["logits"], s["u"], scale=s["scale"], allow=s["allow"], top_k=s["top_k"], top_p=s["top_p"],
                                  min_p=s["min_p"], dtype=TOKENS[case["tokens"]], want_logp=case["logp"], check_status=False)
        return {n: got[n] for n in ("tokens", "logp") if n in got}

    def each(value):
        return value.double().unsqueeze(1) if isinstance(value, torch.Tensor) else value

    x = s["logits"].double()
    if s["allow"] is not None:
        v = torch.arange(V, device=DEVICE)
        x = torch.where(((s["allow"][:, v // 64] >> (v % 64)) & 1).bool(), x, -math.inf)
    m = x.amax(-1, keepdim=True)
    empty = m == -math.inf
    p = torch.exp((x - torch.where(empty, 0.0, m)) * each(s["scale"]))
    if case["rows"] or case["top_k"] or case["top_p"] < 1 or case["min_p"] > 0:
        # the best places first, equal ones by rising place
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices
        best = torch.gather(p, 1, order)
        top_k = each(s["top_k"])
        rank = torch.arange(V, device=DEVICE)
        if case["rows"]:
            best = torch.where((rank < top_k) | (top_k == 0), best, 0.0)
        elif top_k:
            best = torch.where(rank < top_k, best, 0.0)
        upto = best.cumsum(-1)
        ahead = upto - best
        top_p = each(s["top_p"])
        keep = (ahead < top_p * upto[:, -1:]) | (rank == 0)
        if case["rows"]:
            keep = keep | (top_p == 1)
        elif top_p == 1:
            keep = torch.ones_like(keep)
        keep = keep & (best >= each(s["min_p"]))
        p = torch.zeros_like(p).scatter_(1, order, torch.where(keep, best, 0.0))
    upto = p.cumsum(-1)
    tok = torch.searchsorted(upto, s["u"].double() * upto[:, -1:], right=True)
    out = {"tokens": torch.where(empty, -1, tok).to(TOKENS[case["tokens"]])}
    if case["logp"]:
        p_tok = torch.gather(p, 1, tok.clamp(max=V - 1))
        out["logp"] = torch.where(empty, 0.0, torch.log(p_tok / upto[:, -1:])).float()
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "sample":
        R, V, G = case["R"], case["V"], case["G"]
        marks = R * -(-V // 64) * 8 if case["allow"] else 0
        rows = R * (G * (4 + TOKEN_SIZE[case["tokens"]] + 4 * case["logp"]) + 16 * case["rows"])
        return {"bytes": R * V * e + marks + rows, "flops": 6 * R * V + R * G}
    S, H, KV, K, V = (case[n] for n in ("S", "H", "KV", "K", "V"))
    one = H * K + KV * (K + V) + H * V                 # q, k, v and o of a row
    state = 4 * S * H * K * V
    if case["op"] == "step":
        return {"bytes": e * S * one + 2 * state + 4 * S * case["slots"], "flops": 5 * S * H * K * V}
    N = case["N"]
    if not case["train"]:
        return {"bytes": e * N * one + state * (1 + case["h0"]), "flops": 4 * N * H * K * V}
    return {"bytes": 2 * e * N * one + state * (1 + 3 * case["h0"]), "flops": 14 * N * H * K * V}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    wide = {n: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for n, t in s.items()}
    return {"step": _exact_step, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](case, wide)


def _exact_step(case, s):
    group = case["H"] // case["KV"]
    state, o = s["state"].clone(), torch.zeros(case["S"], case["H"], case["V"], dtype=torch.float64, device=DEVICE)
    rows = torch.arange(case["S"], device=DEVICE) if s["slots"] is None else s["slots"].long()
    live = torch.nonzero(rows >= 0)[:, 0]
    for h in range(case["H"]):
        new = s["log_decay"][h].exp() * state[rows[live], h] + torch.einsum("bk,bv->bkv", s["k"][live, h // group], s["v"][live, h // group])
        o[live, h] = s["scale"] * torch.einsum("bk,bkv->bv", s["q"][live, h], new)
        state[rows[live], h] = new
    return {"o": o, "state": state}


def _exact_line(a, into, add, read):
    """One head along all rows, from zero: S_t = a_t S_{t-1} + into_t^T add_t and read_t S_t, row by row in blocks of T rows side by
    side, then block behind block.  Returns what _exact_states needs, and read_t S_t."""
    n, (K, V) = a.shape[0], (into.shape[1], add.shape[1])
    T = max(1, int(math.sqrt(n)))
    B = -(-n // T)
    pad = B * T - n

    def blocks(t, fill):
        return torch.cat([t, t.new_full((pad, *t.shape[1:]), fill)]).view(B, T, *t.shape[1:])

    a, into, add, read = blocks(a, 1.0), blocks(into, 0.0), blocks(add, 0.0), blocks(read, 0.0)

    def walk(state, visit):
        for t in range(T):
            state = a[:, t, None, None] * state + into[:, t, :, None] * add[:, t, None, :]
            visit(t, state)
        return state

    alone = walk(a.new_zeros(B, K, V), lambda t, state: None)
    through = a.prod(1)
    start = torch.zeros_like(alone)
    for b in range(1, B):
        start[b] = through[b - 1] * start[b - 1] + alone[b - 1]
    out = a.new_empty(B, T, V)

    def visit(t, state):
        out[:, t] = (read[:, t, :, None] * state).sum(1)

    walk(start, visit)
    return (walk, start, T), out.view(B * T, V)[:n]


def _exact_states(line, rows):
    """The states at these rows."""
    walk, start, T = line
    found = [None] * len(rows)

    def visit(t, state):
        for i, r in enumerate(rows):
            if r % T == t:
                found[i] = state[r // T].clone()

    walk(start, visit)
    return found


def _exact_attend(case, s):
    N, S, H, K, V, back = (case[n] for n in ("N", "S", "H", "K", "V", "reverse"))
    group, scale = H // case["KV"], s["scale"]
    ptr = [i * (N // S) for i in range(S + 1)] if s["seq_ptr"] is None else s["seq_ptr"].tolist()
    some = [i for i in range(S) if ptr[i + 1] > ptr[i]]
    starts = [ptr[i + 1] - 1 if back else ptr[i] for i in some]
    ends = [ptr[i] if back else ptr[i + 1] - 1 for i in some]
    like = dict(dtype=torch.float64, device=DEVICE)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros(S, H, K, V, **like)
    out = {"o": torch.empty(N, H, V, **like), "last": h0.clone()}
    train = case["train"]
    if train:
        dlast = s["dlast"] if s["dlast"] is not None else torch.zeros(S, H, K, V, **like)
        out.update(dq=torch.empty(N, H, K, **like), dk=torch.zeros(N, case["KV"], K, **like),
                   dv=torch.zeros(N, case["KV"], V, **like), dlog_decay=torch.zeros(H, **like))
        if s["h0"] is not None:
            out["dh0"] = dlast.clone()
    at = torch.arange(N, device=DEVICE)
    length, place, seq_of = (torch.zeros(N, dtype=torch.int64, device=DEVICE) for _ in range(3))
    for i in some:
        length[ptr[i]:ptr[i + 1]], seq_of[ptr[i]:ptr[i + 1]] = ptr[i + 1] - ptr[i], i
        place[ptr[i]:ptr[i + 1]] = (ptr[i + 1] - 1 - at[ptr[i]:ptr[i + 1]]) if back else at[ptr[i]:ptr[i + 1]] - ptr[i]

    def line(a, into, add, read, backwards):
        f = (lambda t: t.flip(0)) if backwards else (lambda t: t)
        kept, got = _exact_line(f(a), f(into), f(add), f(read))
        return (lambda rows: _exact_states(kept, [N - 1 - r for r in rows] if backwards else rows)), f(got)

    for h in range(H):
        gamma = s["log_decay"][h].exp()
        q, k, v = s["q"][:, h], s["k"][:, h // group], s["v"][:, h // group]
        # what a sequence begins with counts as decayed by its rows' places
        a = torch.full((N,), 1.0, **like) * gamma
        a[starts] = 0
        worn = gamma ** (place + 1).double()
        find, o = line(a, k, v, q, back)
        own_h0 = h0[:, h]
        for j, i in enumerate(some):
            rows = slice(ptr[i], ptr[i + 1])
            o[rows] += worn[rows, None] * (q[rows] @ own_h0[i])
        out["o"][:, h] = scale * o
        for i, e, state in zip(some, ends, find(ends)):
            out["last"][i, h] = state + worn[e] * own_h0[i]
        if not train:
            continue
        do = s["do"][:, h]
        _, dq = line(a, v, k, do, back)
        a = torch.full((N,), 1.0, **like) * gamma
        a[ends] = 0
        left = gamma ** (length - 1 - place).double()      # from a row to its sequence's end
        find, dv = line(a, scale * q, do, k, not back)
        _, dk = line(a, scale * do, q, v, not back)
        for i in some:
            rows = slice(ptr[i], ptr[i + 1])
            dq[rows] += worn[rows, None] * (do[rows] @ own_h0[i].T)
            dv[rows] += left[rows, None] * (k[rows] @ dlast[i, h])
            dk[rows] += left[rows, None] * (v[rows] @ dlast[i, h].T)
        dq = scale * dq
        out["dq"][:, h] = dq
        out["dk"][:, h // group] += dk
        out["dv"][:, h // group] += dv
        # <D_t, gamma S_{t-1}> falls from row to row by what q and k have of the gradient
        step = (q * dq).sum(-1) - (k * dk).sum(-1)
        total = ((place + 1) * step).sum()
        for i in some:
            total += (ptr[i + 1] - ptr[i]) * (dlast[i, h] * out["last"][i, h]).sum()
        out["dlog_decay"][h] = total
        if s["h0"] is not None:
            for i, b, state in zip(some, starts, find(starts)):
                out["dh0"][i, h] = gamma * state + worn[ends[some.index(i)]] * dlast[i, h]
    return out


def _exact_sample(case, s):
    R, V, G = case["R"], case["V"], case["G"]
    u = s["u"]
    column = lambda v: v.view(R, 1) if isinstance(v, torch.Tensor) else torch.full((R, 1), v, device=DEVICE)  # noqa: E731
    bit = torch.arange(64, device=DEVICE)
    open_ = torch.ones(R, V, dtype=torch.bool, device=DEVICE)
    if s["allow"] is not None:
        open_ = ((s["allow"].unsqueeze(-1) >> bit) & 1).view(R, -1)[:, :V].bool()
    empty = ~open_.any(-1, keepdim=True)
    x = s["logits"].masked_fill(~open_, -math.inf)
    lp = torch.log_softmax(torch.where(empty, 0.0, x * column(s["scale"])), -1)
    # a place's rank among the row's, and what the places in front of it have together
    sinking = torch.argsort(-x, dim=-1, stable=True)
    rank = torch.argsort(sinking, dim=-1)
    top_k = column(s["top_k"])
    kept = (rank < torch.where(top_k == 0, V, top_k)) & open_
    top_p = column(s["top_p"])
    if bool((top_p < 1).any()):
        share = torch.where(kept, lp.exp(), 0.0)
        ranked = torch.gather(share, 1, sinking)
        front = torch.gather(torch.cat([torch.zeros_like(ranked[:, :1]), ranked.cumsum(-1)[:, :-1]], 1), 1, rank)
        kept &= (front < top_p * share.sum(-1, keepdim=True)) | (top_p == 1)
    kept &= (lp - lp.amax(-1, keepdim=True)).exp() >= column(s["min_p"])
    lp = torch.where(kept, lp, -math.inf)
    lp = lp - torch.where(empty, 0.0, torch.logsumexp(lp, -1, keepdim=True))
    upto = lp.exp().cumsum(-1)
    if V <= 64:
        tok = torch.zeros(R, G, dtype=torch.int64, device=DEVICE)
        for v in range(V - 1):
            tok += u >= upto[:, v:v + 1]
    else:
        tok = torch.searchsorted(upto, u, right=True).clamp(max=V - 1)
    out = {"tokens": torch.where(empty, -1, tok).to(TOKENS[case["tokens"]])}
    if case["logp"]:
        out["logp"] = torch.where(empty, 0.0, torch.gather(lp, 1, tok))
    return out
