"""Linear attention with a decay for each head on torch tensors (see ``include/cpeval.h``).

``cp_linear_attention`` (with ``_backward`` and ``_step``) follows the C entry points of the same names, in the manner of
``policy``: arguments are checked, outputs and workspaces allocated, and the library's kernels called on ``stream``.
Inputs may be views with any distance from row to row and from head to head (slices of a fused projection, heads in
front of rows, expanded heads), as long as a head's elements are contiguous.
"""
from __future__ import annotations

import ctypes as C
import functools

from .binding import CpError, load_library
from .policy import (STATUS_BAD_SEQUENCE, STATUS_BAD_SLOT, _check, _need, _on_gpu, _place, _room, _type, _vector, _vector_out)


def _heads(t, name, lead, heads, width, dtype, device):
    """(address, distance of rows, distance of heads) of a [..][heads][width] tensor."""
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype}, not {t.dtype}")
    if t.shape != (*lead, heads, width):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, not {(*lead, heads, width)}")
    stride = t.stride()
    if width > 1 and stride[-1] != 1:
        raise ValueError(f"{name}: the elements of a head have to be contiguous (strides {tuple(stride)})")
    ld = stride[-3] if len(lead) == 1 or lead[1] > 1 else stride[0]
    if len(lead) == 2 and lead[0] > 1 and lead[1] > 1 and stride[0] != lead[1] * ld:
        raise ValueError(f"{name}: all rows have to be equally far apart (strides {tuple(stride)})")
    # (what has a single row or head is at no distance from another)
    rows = lead[0] if len(lead) == 1 else lead[0] * lead[1]
    return t.data_ptr(), ld if rows > 1 else heads * width, stride[-2] if heads > 1 else width


def _heads_out(out, key, lead, heads, width, dtype, device):
    import torch
    t = out.get(key)
    if t is None:
        t = out[key] = torch.empty((*lead, heads, width), dtype=dtype, device=device)
        return t.data_ptr(), heads * width, width
    return _heads(t, key, lead, heads, width, dtype, device)


def _shape(q, k, v, seq_ptr, device):
    """(leading axes, rows, sequences, address of seq_ptr, heads, kv_heads, width_k, width_v)"""
    import torch
    if q.dim() not in (3, 4) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError(f"q, k, v: [rows][heads][width] or [batch][rows][heads][width], not {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}")
    lead = tuple(q.shape[:-2])
    heads, kv_heads = int(q.shape[-2]), int(k.shape[-2])
    if kv_heads < 1 or heads % kv_heads:
        raise ValueError(f"{heads} heads cannot share {kv_heads} heads of keys and values")
    rows = lead[0] if len(lead) == 1 else lead[0] * lead[1]
    sizes = heads, kv_heads, int(q.shape[-1]), int(v.shape[-1])
    if seq_ptr is None:
        return lead, rows, 1 if len(lead) == 1 else lead[0], None, sizes
    if len(lead) == 2:
        raise ValueError("seq_ptr: with packed rows [rows][heads][width] only")
    if seq_ptr.device != device or seq_ptr.dtype != torch.int32 or seq_ptr.dim() != 1 or not seq_ptr.is_contiguous():
        raise ValueError("seq_ptr: a contiguous int32 tensor [sequences + 1] on the device of q")
    return lead, rows, int(seq_ptr.shape[0]) - 1, seq_ptr.data_ptr(), sizes


@functools.lru_cache(maxsize=4096)
def _carry_states(rows, count, packed, heads, wk, wv):
    found = C.c_int64(0)
    rc = load_library().cp_linear_attention_carry_states(rows, count, packed, heads, wk, wv, C.byref(found))
    if rc:
        raise CpError(rc, "cp_linear_attention_carry_states")
    return int(found.value)


def cp_linear_attention(q, k, v, log_decay=None, *, scale=1.0, seq_ptr=None, h0=None, reverse=False, want_last=False, want_carry=False,
                        out=None, workspace=None, stream=None, check_status=True):
    """o_t = scale q_t S_t with S_t = exp(log_decay) S_{t-1} + k_t^T v_t, per head.

    ``q`` [rows][heads][width_k], ``k`` [rows][kv_heads][width_k], ``v`` [rows][kv_heads][width_v]: one sequence or those that
    ``seq_ptr`` (int32 [sequences + 1]; rows behind its last entry are left alone) cuts the rows into, or with a batch axis in
    front, ``batch`` sequences.  heads / kv_heads neighbouring heads share keys and values.  ``log_decay`` float32 [heads], at most
    0; ``h0`` float32 [sequences][heads][width_k][width_v].  Returns a dict: ``o`` [..][heads][width_v]; ``last`` as ``h0`` if
    wanted; ``carry`` if wanted (what cp_linear_attention_backward needs); ``status`` with ``seq_ptr``.  With ``check_status`` and
    ``seq_ptr`` the stream is synchronised and bad pointers raise."""
    import torch
    lib = load_library()
    dev = _on_gpu(q, "q")
    lead, rows, count, ptr, sizes = _shape(q, k, v, seq_ptr, dev)
    heads, kv_heads, wk, wv = sizes
    kind, dt, f32 = _type(q, "q"), q.dtype, torch.float32
    ins = (*_heads(q, "q", lead, heads, wk, dt, dev), *_heads(k, "k", lead, kv_heads, wk, dt, dev), *_heads(v, "v", lead, kv_heads, wv, dt, dev))
    decay_at, state = _vector(log_decay, "log_decay", (heads,), f32, dev), (count, heads, wk, wv)
    h0_at = _vector(h0, "h0", state, f32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        o = _heads_out(out, "o", lead, heads, wv, dt, dev)
        last_at = _vector_out(out, "last", state, f32, dev) if want_last or "last" in out else None
        carry_at = None
        if want_carry or "carry" in out:
            carry_at = _vector_out(out, "carry", (_carry_states(rows, count, ptr is not None, heads, wk, wv), heads, wk, wv), f32, dev) or None
        status_at = _vector_out(out, "status", (1,), torch.int32, dev) if ptr is not None else None
        work, work_at, room = _room(workspace, _need("cp_linear_attention_workspace_bytes", rows, count, ptr is not None, *sizes, 0), dev)
        rc = lib.cp_linear_attention(rows, count, ptr, *sizes, kind, int(bool(reverse)), *ins, decay_at, scale, h0_at, *o, last_at, carry_at,
                                     work_at, room, handle, status_at)
    if rc:
        raise CpError(rc, "cp_linear_attention")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to at most the number of rows", stream)
    return out


def cp_linear_attention_backward(do, q, k, v, log_decay, carry, *, dlast=None, scale=1.0, seq_ptr=None, h0=None, reverse=False, out=None,
                                 workspace=None, stream=None, check_status=True):
    """Gradient of cp_linear_attention for the same inputs and the ``carry`` of that call.  Returns a dict: ``dq``, ``dk``,
    ``dv`` as ``q``, ``k`` and ``v``, ``dlog_decay`` float32 [heads] with ``log_decay``, ``dh0`` with ``h0``."""
    import torch
    lib = load_library()
    dev = _on_gpu(q, "q")
    lead, rows, count, ptr, sizes = _shape(q, k, v, seq_ptr, dev)
    heads, kv_heads, wk, wv = sizes
    kind, dt, f32 = _type(q, "q"), q.dtype, torch.float32
    d_o = _heads(do, "do", lead, heads, wv, dt, dev)
    ins = (*_heads(q, "q", lead, heads, wk, dt, dev), *_heads(k, "k", lead, kv_heads, wk, dt, dev), *_heads(v, "v", lead, kv_heads, wv, dt, dev))
    decay_at, state = _vector(log_decay, "log_decay", (heads,), f32, dev), (count, heads, wk, wv)
    h0_at, dlast_at = _vector(h0, "h0", state, f32, dev), _vector(dlast, "dlast", state, f32, dev)
    carry_at = _vector(carry, "carry", (_carry_states(rows, count, ptr is not None, heads, wk, wv), heads, wk, wv), f32, dev) or None
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        dq, dk, dv = (_heads_out(out, "dq", lead, heads, wk, dt, dev), _heads_out(out, "dk", lead, kv_heads, wk, dt, dev),
                      _heads_out(out, "dv", lead, kv_heads, wv, dt, dev))
        dd_at = _vector_out(out, "dlog_decay", (heads,), f32, dev) if log_decay is not None or "dlog_decay" in out else None
        dh0_at = _vector_out(out, "dh0", state, f32, dev) if h0 is not None or "dh0" in out else None
        status_at = _vector_out(out, "status", (1,), torch.int32, dev) if ptr is not None else None
        work, work_at, room = _room(workspace, _need("cp_linear_attention_workspace_bytes", rows, count, ptr is not None, *sizes, 1), dev)
        rc = lib.cp_linear_attention_backward(rows, count, ptr, *sizes, kind, int(bool(reverse)), *d_o, dlast_at, *ins, decay_at, scale,
                                              h0_at, carry_at, *dq, *dk, *dv, dd_at, dh0_at, work_at, room, handle, status_at)
    if rc:
        raise CpError(rc, "cp_linear_attention_backward")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to at most the number of rows", stream)
    return out


def cp_linear_attention_step(q, k, v, state, log_decay=None, *, scale=1.0, slots=None, out=None, stream=None, check_status=True):
    """One more row of every sequence: ``q`` [sequences][heads][width_k], ``k``, ``v`` with their heads; ``state`` float32
    [slots][heads][width_k][width_v] is updated in place, row ``slots[i]`` (int32, all different; negative: none) for
    sequence i, or row i.  Returns a dict: ``o`` [sequences][heads][width_v], ``status`` with ``slots``."""
    import torch
    lib = load_library()
    dev = _on_gpu(q, "q")
    if q.dim() != 3 or state.dim() != 4:
        raise ValueError("q: [sequences][heads][width_k], state: [slots][heads][width_k][width_v]")
    lead, count, _, _, sizes = _shape(q, k, v, None, dev)
    heads, kv_heads, wk, wv = sizes
    kind, dt, f32, i32 = _type(q, "q"), q.dtype, torch.float32, torch.int32
    ins = (*_heads(q, "q", lead, heads, wk, dt, dev), *_heads(k, "k", lead, kv_heads, wk, dt, dev), *_heads(v, "v", lead, kv_heads, wv, dt, dev))
    num_slots = int(state.shape[0])
    decay_at = _vector(log_decay, "log_decay", (heads,), f32, dev)
    state_at, slots_at = _vector(state, "state", (num_slots, heads, wk, wv), f32, dev), _vector(slots, "slots", (count,), i32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        o = _heads_out(out, "o", lead, heads, wv, dt, dev)
        status_at = _vector_out(out, "status", (1,), i32, dev) if slots is not None else None
        rc = lib.cp_linear_attention_step(count, *sizes, kind, *ins, decay_at, scale, state_at, num_slots, slots_at, *o, handle, status_at)
    if rc:
        raise CpError(rc, "cp_linear_attention_step")
    if check_status and slots is not None:
        _check(out["status"], STATUS_BAD_SLOT, "a slot lies behind the last state", stream)
    return out
