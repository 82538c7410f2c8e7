"""A placement policy that is trained by the critical-path times of the partitions it draws.

    python examples/learn_placement.py --workload inception --steps 100

The vertices of a data-flow graph are read in topological order.  Each block of the policy is

    z  = norm(x + gate * norm(y))      the joint with the block before             (norm_gate)
    f, v, gate = slices of z @ W       one product of the library
    y  = recurrence(f, v) @ U          a vertex sees those before it               (recurrence)

and the head gives every vertex a row of logits over the devices.  A step draws partitions from the rows,
``cp_eval`` rates them, and the log probabilities of what was drawn (token_logprobs), weighted by the ratings
and with the rows' entropy added, are the loss.  ``place`` runs the trained policy vertex by vertex
(cp_recurrence_step), as a program does that places a graph while it is being built.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_1711_01912_amd as cpe  # noqa: E402
from paper_1711_01912_amd import autograd  # noqa: E402
from paper_1711_01912_amd.binding import ASSIGN_VERTEX_MAJOR  # noqa: E402


def features(w):
    """[n][6] floats, vertices in topological order; the order itself."""
    order = np.asarray(w.level_vtx, dtype=np.int64)
    out_deg, in_deg = np.diff(w.succ_ptr), np.diff(w.pred_ptr)
    volume = np.bincount(np.repeat(np.arange(w.n), out_deg), weights=w.succ_t, minlength=w.n)
    cols = [np.log1p(w.c), np.log1p(volume), np.log1p(out_deg), np.log1p(in_deg), w.level / max(1, w.L - 1)]
    table = np.stack([np.asarray(c, dtype=np.float64) for c in cols], 1)
    table = (table - table.mean(0)) / (table.std(0) + 1e-6)
    table = np.concatenate([table, np.ones((w.n, 1))], 1)
    return torch.from_numpy(table[order]).float(), torch.from_numpy(order)


class Policy(torch.nn.Module):
    def __init__(self, devices, width=128, blocks=2, dtype=torch.bfloat16, inputs=6, seed=0):
        super().__init__()
        g = torch.Generator().manual_seed(seed)

        def matrix(rows, cols, by=1.0):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=g) * by / rows ** 0.5).to(dtype))

        self.dtype, self.blocks, self.width = dtype, blocks, width
        self.embed = matrix(inputs, width)
        self.into = torch.nn.ParameterList(matrix(width, 3 * width) for _ in range(blocks))
        self.back = torch.nn.ParameterList(matrix(width, width) for _ in range(blocks))
        # time scales from two vertices to a few hundred
        self.bias = torch.nn.ParameterList(torch.nn.Parameter(torch.linspace(0, 5, width)) for _ in range(blocks))
        self.w_pre = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(width)) for _ in range(blocks + 1))
        self.w_post = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(width)) for _ in range(blocks))
        self.head = matrix(width, devices, by=0.1)

    def forward(self, inputs):
        """Logits [n][devices] of the vertices with these inputs, in their order."""
        x, y, gate = (inputs.to(self.dtype) @ self.embed).float(), None, None
        for i in range(self.blocks):
            x, z = self._joint(autograd.norm_gate, i, x, y, gate)
            f, v, gate = (z @ self.into[i]).split(self.width, 1)
            h, _ = autograd.recurrence(f, v, bias=self.bias[i])
            y = h @ self.back[i]
        return self._joint(autograd.norm_gate, self.blocks, x, y, gate)[1] @ self.head

    def _joint(self, norm_gate, i, x, y, gate):
        if i == 0:
            return norm_gate(x, w_pre=self.w_pre[0], z_dtype=self.dtype)
        return norm_gate(x, y, gate, w_pre=self.w_pre[i], w_post=self.w_post[i - 1], gate_act="silu", scale=0.5)

    @torch.no_grad()
    def step(self, inputs, states):
        """Logits [sequences][devices] of one more vertex of each sequence; ``states``: float32 [blocks][sequences][width],
        updated in place."""
        def joint(x, y=None, gate=None, **kw):
            out = cpe.cp_norm_gate(x, y, gate, **kw)
            return out.get("r", x), out["z"]

        x, y, gate = (inputs.to(self.dtype) @ self.embed).float(), None, None
        for i in range(self.blocks):
            x, z = self._joint(joint, i, x, y, gate)
            f, v, gate = (z @ self.into[i]).split(self.width, 1)
            h = cpe.cp_recurrence_step(f, v, states[i], bias=self.bias[i], check_status=False)["h"]
            y = h @ self.back[i]
        return self._joint(joint, self.blocks, x, y, gate)[1] @ self.head


def draw(logits, partitions, generator=None):
    """uint8 [n][partitions]"""
    return torch.multinomial(logits.float().softmax(-1), partitions, replacement=True, generator=generator).to(torch.uint8)


def rate(graph, w, order, tokens):
    """Critical-path time of every partition, float64 [partitions]."""
    assignments = torch.empty_like(tokens)
    assignments[order] = tokens          # (from topological order to the vertices' numbers)
    out = cpe.cp_eval(graph, assignments, w.speeds, w.bandwidth, want=("cp",), assign_layout=ASSIGN_VERTEX_MAJOR)
    return out["cp"].double()


def train(w, steps=100, partitions=256, width=128, blocks=2, lr=3e-3, dtype=torch.bfloat16, seed=0, say=None):
    """(policy, mean critical-path time of each step's partitions, best partition's time)"""
    device = torch.device("cuda:0")
    graph = cpe.CpGraph.from_workload(w, device="cuda:0")
    inputs, order = (t.to(device) for t in features(w))
    policy = Policy(w.k, width, blocks, dtype, seed=seed).to(device)
    generator = torch.Generator(device=device)
    generator.manual_seed(seed)
    optimizer = torch.optim.Adam(policy.parameters(), lr=lr)
    history, best = [], float("inf")
    for step in range(steps):
        logits = policy(inputs)
        tokens = draw(logits.detach(), partitions, generator)
        cp = rate(graph, w, order, tokens)
        gain = ((cp.mean() - cp) / (cp.std() + 1e-9)).float()
        logp, entropy = autograd.token_logprobs(logits, tokens)
        loss = -(logp * gain).sum() / partitions - 1e-3 * entropy.sum()
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        history.append(float(cp.mean()))
        best = min(best, float(cp.min()))
        if say and (step % 10 == 0 or step + 1 == steps):
            say(f"step {step}: mean critical path {history[-1]:.0f}, best partition so far {best:.0f}")
    return policy, history, best


def place(policy, w):
    """The policy's most likely device of every vertex, uint8 [n], vertex by vertex."""
    device = policy.head.device
    inputs, order = (t.to(device) for t in features(w))
    states = torch.zeros(policy.blocks, 1, policy.width, device=device)
    found = torch.empty(w.n, dtype=torch.uint8, device=device)
    for t in range(w.n):
        logits = policy.step(inputs[t:t + 1], states)
        found[t] = cpe.cp_token_logprobs(logits, top=1, check_status=False)["top_idx"][0, 0]
    tokens = torch.empty_like(found)
    tokens[order] = found
    return tokens


def main():
    from workloads import CONFIG_NAMES, make_workload
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="inception", choices=CONFIG_NAMES)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--partitions", type=int, default=256)
    args = ap.parse_args()
    w = make_workload(args.workload)
    policy, _, best = train(w, args.steps, args.partitions, say=print)
    if w.n <= 10000:
        tokens = place(policy, w)
        graph = cpe.CpGraph.from_workload(w, device="cuda:0")
        cp = cpe.cp_eval(graph, tokens.view(1, -1), w.speeds, w.bandwidth, want=("cp",))["cp"]
        print(f"placed vertex by vertex: critical path {int(cp[0])} (best drawn partition {best:.0f})")


if __name__ == "__main__":
    main()
