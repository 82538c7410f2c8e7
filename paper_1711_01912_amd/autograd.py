"""The operators of a learned placement policy as differentiable functions of torch tensors.

``recurrence``, ``norm_gate`` and ``token_logprobs`` call the forward entry points of ``policy`` and, when a
gradient is asked for, the backward ones; what these need is kept by the graph as usual.  Everything runs on the
current stream.  Pointers and tokens are told to be bad by ``policy``'s own calls with ``check_status``; here
nothing is synchronised, and so the functions may be captured into a HIP graph.  (A backward pass is captured
while no eager graph of the same leaves is alive: torch would join the capture with the stream that such a graph
ran on.)  Gradients of second order are not there.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import policy


def _rows(grad, like):
    """A gradient as the kernels read it: rows of contiguous elements, zeros where there is none."""
    if grad is None:
        return torch.zeros_like(like, memory_format=torch.contiguous_format)
    return grad.contiguous()


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, f, x, bias, h0, seq_ptr, reverse):
        kw = dict(bias=bias, h0=h0, seq_ptr=seq_ptr, reverse=reverse, check_status=False)
        out = policy.cp_recurrence(f, x, want_last=True, want_carry=any(ctx.needs_input_grad), **kw)
        ctx.save_for_backward(f, x, bias, h0, seq_ptr, out.get("carry"))
        ctx.reverse = reverse
        ctx.set_materialize_grads(False)
        return out["h"], out["last"]

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dlast):
        f, x, bias, h0, seq_ptr, carry = ctx.saved_tensors
        out = policy.cp_recurrence_backward(_rows(dh, x), f, x, carry, dlast=None if dlast is None else dlast.contiguous(),
                                            bias=bias, seq_ptr=seq_ptr, h0=h0, reverse=ctx.reverse, check_status=False)
        return out["df"], out["dx"], out.get("dbias"), out.get("dh0"), None, None


def recurrence(f, x, *, bias=None, h0=None, seq_ptr=None, reverse=False):
    """(h, last) of policy.cp_recurrence, differentiable in f, x, bias and h0."""
    return _Recurrence.apply(f, x, bias, h0, seq_ptr, reverse)


class _NormGate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, gate, w_pre, w_post, gate_act, scale, eps, z_dtype):
        out = policy.cp_norm_gate(x, y, gate, w_pre=w_pre, w_post=w_post, gate_act=gate_act, scale=scale, eps=eps,
                                  z_dtype=z_dtype, want_stats=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, y, gate, w_pre, w_post, out.get("stats"))
        ctx.options = dict(gate_act=gate_act, scale=scale)
        ctx.z_dtype = out["z"].dtype
        ctx.set_materialize_grads(False)
        return out["z"], out.get("r")

    @staticmethod
    @once_differentiable
    def backward(ctx, dz, dr):
        x, y, gate, w_pre, w_post, stats = ctx.saved_tensors
        dz = torch.zeros(x.shape, dtype=ctx.z_dtype, device=x.device) if dz is None else dz.contiguous()
        out = policy.cp_norm_gate_backward(None if dr is None else dr.contiguous(), dz, x, y, gate, w_pre=w_pre, w_post=w_post,
                                           stats=stats, **ctx.options)
        return out["dx"], out.get("dy"), out.get("dgate"), out["dw_pre"], out.get("dw_post"), None, None, None, None


def norm_gate(x, y=None, gate=None, *, w_pre, w_post=None, gate_act="sigmoid", scale=1.0, eps=1e-6, z_dtype=None):
    """(r, z) of policy.cp_norm_gate (r is x without y), differentiable in x, y, gate, w_pre and w_post."""
    z, r = _NormGate.apply(x, y, gate, w_pre, w_post, gate_act, scale, eps, z_dtype)
    return (x if y is None else r), z


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, allow, scale):
        out = policy.cp_token_logprobs(logits, tokens, scale=scale, allow=allow, check_status=False)
        ctx.save_for_backward(logits, tokens, allow, out["stats"])
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out.get("logp"), out["entropy"]

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dentropy):
        logits, tokens, allow, stats = ctx.saved_tensors
        if dlogp is None:        # only the entropy's
            tokens = None
        out = policy.cp_token_logprobs_backward(logits, tokens, stats, dlogp, dentropy=dentropy, scale=ctx.scale, allow=allow)
        return out["dlogits"], None, None, None


def token_logprobs(logits, tokens, *, scale=1.0, allow=None):
    """(logp, entropy) of policy.cp_token_logprobs, differentiable in the logits."""
    return _TokenLogprobs.apply(logits, tokens, allow, scale)
