"""The operators of a learned placement policy on torch tensors (see ``include/cpeval.h``).

``cp_recurrence`` (with ``_backward`` and ``_step``), ``cp_norm_gate`` (with ``_backward``) and
``cp_token_logprobs`` (with ``_backward``) follow the C entry points of the same names.  As in
``binding``, nothing is computed here: arguments are checked, outputs and workspaces allocated, and
the library's kernels called on ``stream`` (default: the current one).  Outputs and workspaces are
allocated for that stream; inputs that another stream still writes are the caller's to wait for.
Matrices may be views whose rows are further apart than their length (slices of a fused
projection), as long as a row's elements are contiguous.  ``out`` may carry preallocated outputs
under the keys of the result, ``workspace`` a preallocated uint8 tensor.

``autograd`` has the same operators as differentiable functions.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools

from .binding import CpError, load_library

TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
GATE_NONE, GATE_SIGMOID, GATE_SILU = 0, 1, 2
GATES = {"none": GATE_NONE, "sigmoid": GATE_SIGMOID, "silu": GATE_SILU}
STATUS_BAD_TOKEN, STATUS_BAD_SEQUENCE, STATUS_BAD_SLOT = 32, 64, 128
RECURRENCE_CHUNK = 128


@functools.lru_cache(maxsize=1)
def _types():
    import torch
    return {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}


def _type(t, name):
    code = _types().get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: float32, bfloat16 or float16, not {t.dtype}")
    return code


def _matrix(t, name, rows, width, dtype, device):
    """The distance between the rows of a [rows][width] (or [batch][rows / batch][width]) tensor."""
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype}, not {t.dtype}")
    shape, stride = t.shape, t.stride()
    if shape[-1] != width or t.numel() != rows * width:
        raise ValueError(f"{name}: shape {tuple(shape)} does not fit {rows} rows of {width}")
    if t.numel() == 0:
        return width
    if width > 1 and stride[-1] != 1:
        raise ValueError(f"{name}: the elements of a row have to be contiguous (strides {tuple(stride)})")
    if len(shape) == 3 and shape[0] > 1 and shape[1] > 1 and stride[0] != shape[1] * stride[1]:
        raise ValueError(f"{name}: all rows have to be equally far apart (strides {tuple(stride)})")
    if rows == 1:
        return width
    ld = stride[0] if len(shape) == 2 or shape[1] == 1 else stride[1]
    if ld < width:
        raise ValueError(f"{name}: rows overlap (strides {tuple(stride)})")
    return ld


def _vector(t, name, shape, dtype, device):
    """The address of a contiguous tensor of that shape, or None."""
    if t is None:
        return None
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype}, not {t.dtype}")
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of shape {shape}, not {tuple(t.shape)}")
    return t.data_ptr()


def _on_gpu(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} has to be on the GPU")
    return t.device


@contextlib.contextmanager
def _other(device, stream):
    import torch
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield


def _place(device, stream):
    """What to allocate and launch under, and the stream's handle."""
    import torch
    if stream is None and device.index == torch.cuda.current_device():
        return contextlib.nullcontext(), torch.cuda.current_stream().cuda_stream
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        raise ValueError(f"the stream is {stream.device}'s, the tensors are on {device}")
    return _other(device, stream), stream.cuda_stream


@functools.lru_cache(maxsize=4096)
def _need(entry, *sizes):
    out = C.c_size_t(0)
    rc = getattr(load_library(), entry)(*sizes, C.byref(out))
    if rc:
        raise CpError(rc, entry)
    return int(out.value)


def _work(workspace, need, device):
    import torch
    if workspace is None:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=device) if need else None
    if workspace.device != device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous uint8 tensor on the device of the inputs")
    return workspace


def _room(work):
    return (None, 0) if work is None else (work.data_ptr(), work.numel())


def _check(status, flag, text, device):
    import torch
    torch.cuda.synchronize(device)
    if int(status.item()) & flag:
        raise ValueError(text)


# ---- recurrence ------------------------------------------------------------------------------------


def _sequences(f, seq_ptr, device):
    import torch
    if f.dim() not in (2, 3):
        raise ValueError(f"f: [rows][width] or [batch][rows][width], not {tuple(f.shape)}")
    width = int(f.shape[-1])
    rows = int(f.shape[0]) if f.dim() == 2 else int(f.shape[0] * f.shape[1])
    if seq_ptr is None:
        return rows, width, 1 if f.dim() == 2 else int(f.shape[0]), None
    if f.dim() == 3:
        raise ValueError("seq_ptr: with packed rows [rows][width] only")
    if seq_ptr.device != device or seq_ptr.dtype != torch.int32 or seq_ptr.dim() != 1 or not seq_ptr.is_contiguous():
        raise ValueError("seq_ptr: a contiguous int32 tensor [sequences + 1] on the device of f")
    return rows, width, int(seq_ptr.shape[0]) - 1, seq_ptr.data_ptr()


def cp_recurrence(f, x, *, bias=None, seq_ptr=None, h0=None, reverse=False, want_last=False, want_carry=False, out=None,
                  workspace=None, stream=None, check_status=True):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f + bias), per channel.

    ``f``, ``x``: [rows][width], one sequence or those that ``seq_ptr`` (int32 [sequences + 1]) cuts the rows
    into, or [batch][rows][width], ``batch`` sequences.  ``bias`` float32 [width]; ``h0`` float32
    [sequences][width].  Returns a dict: ``h`` as ``x``; ``last`` float32 [sequences][width] if wanted;
    ``carry`` if wanted (what cp_recurrence_backward needs); ``status`` with ``seq_ptr``.  With
    ``check_status`` and ``seq_ptr`` the stream is synchronised and bad pointers raise."""
    import torch
    lib = load_library()
    dev = _on_gpu(f, "f")
    rows, width, count, ptr = _sequences(f, seq_ptr, dev)
    kind, f32 = _type(f, "f"), torch.float32
    ldf, ldx = _matrix(f, "f", rows, width, f.dtype, dev), _matrix(x, "x", rows, width, f.dtype, dev)
    if x.shape != f.shape:
        raise ValueError("f and x have different shapes")
    bias_at, h0_at = _vector(bias, "bias", (width,), f32, dev), _vector(h0, "h0", (count, width), f32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        if "h" not in out:
            out["h"] = torch.empty(x.shape, dtype=x.dtype, device=dev)
        if want_last and "last" not in out:
            out["last"] = torch.empty((count, width), dtype=f32, device=dev)
        if want_carry and "carry" not in out:
            out["carry"] = torch.empty((-(-rows // RECURRENCE_CHUNK), width), dtype=f32, device=dev)
        if ptr is not None and "status" not in out:
            out["status"] = torch.empty(1, dtype=torch.int32, device=dev)
        work = _work(workspace, _need("cp_recurrence_workspace_bytes", rows, width, 0) if rows > RECURRENCE_CHUNK else 0, dev)
        ldh = _matrix(out["h"], "h", rows, width, f.dtype, dev)
        rc = lib.cp_recurrence(rows, width, count, ptr, kind, int(bool(reverse)), f.data_ptr(), ldf, x.data_ptr(), ldx, bias_at,
                               h0_at, out["h"].data_ptr(), ldh, _vector(out.get("last"), "last", (count, width), f32, dev),
                               _vector(out.get("carry"), "carry", (-(-rows // RECURRENCE_CHUNK), width), f32, dev), *_room(work),
                               handle, _vector(out.get("status"), "status", (1,), torch.int32, dev))
    if rc:
        raise CpError(rc, "cp_recurrence")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to the number of rows", dev)
    return out


def cp_recurrence_backward(dh, f, x, carry, *, dlast=None, bias=None, seq_ptr=None, h0=None, reverse=False, out=None,
                           workspace=None, stream=None, check_status=True):
    """Gradient of cp_recurrence for the same inputs and the ``carry`` of that call.  Returns a dict: ``df``, ``dx`` as
    ``f`` and ``x``, ``dbias`` float32 [width] with ``bias``, ``dh0`` float32 [sequences][width] with ``h0``."""
    import torch
    lib = load_library()
    dev = _on_gpu(f, "f")
    rows, width, count, ptr = _sequences(f, seq_ptr, dev)
    kind, f32 = _type(f, "f"), torch.float32
    lds = [_matrix(t, n, rows, width, f.dtype, dev) for t, n in ((dh, "dh"), (f, "f"), (x, "x"))]
    bias_at, h0_at = _vector(bias, "bias", (width,), f32, dev), _vector(h0, "h0", (count, width), f32, dev)
    dlast_at = _vector(dlast, "dlast", (count, width), f32, dev)
    carry_at = _vector(carry, "carry", (-(-rows // RECURRENCE_CHUNK), width), f32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        for key, like in (("df", f), ("dx", x)):
            if key not in out:
                out[key] = torch.empty(like.shape, dtype=like.dtype, device=dev)
        if bias is not None and "dbias" not in out:
            out["dbias"] = torch.empty(width, dtype=f32, device=dev)
        if h0 is not None and "dh0" not in out:
            out["dh0"] = torch.empty((count, width), dtype=f32, device=dev)
        if ptr is not None and "status" not in out:
            out["status"] = torch.empty(1, dtype=torch.int32, device=dev)
        work = _work(workspace, _need("cp_recurrence_workspace_bytes", rows, width, 1), dev)
        lddf, lddx = (_matrix(out[k], k, rows, width, f.dtype, dev) for k in ("df", "dx"))
        rc = lib.cp_recurrence_backward(rows, width, count, ptr, kind, int(bool(reverse)), dh.data_ptr(), lds[0], dlast_at,
                                        f.data_ptr(), lds[1], x.data_ptr(), lds[2], bias_at, h0_at, carry_at,
                                        out["df"].data_ptr(), lddf, out["dx"].data_ptr(), lddx,
                                        _vector(out.get("dbias"), "dbias", (width,), f32, dev),
                                        _vector(out.get("dh0"), "dh0", (count, width), f32, dev), *_room(work), handle,
                                        _vector(out.get("status"), "status", (1,), torch.int32, dev))
    if rc:
        raise CpError(rc, "cp_recurrence_backward")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to the number of rows", dev)
    return out


def cp_recurrence_step(f, x, state, *, bias=None, slots=None, out=None, stream=None, check_status=True):
    """One more row of every sequence: ``f``, ``x`` [sequences][width]; ``state`` float32 [slots][width] is updated in
    place, row ``slots[i]`` (int32, all different; negative: none) for sequence i, or row i.  Returns a dict: ``h`` as
    ``x``, ``status`` with ``slots``."""
    import torch
    lib = load_library()
    dev = _on_gpu(f, "f")
    if f.dim() != 2 or state.dim() != 2:
        raise ValueError("f: [sequences][width], state: [slots][width]")
    count, width = int(f.shape[0]), int(f.shape[1])
    kind, f32, i32 = _type(f, "f"), torch.float32, torch.int32
    ldf, ldx = _matrix(f, "f", count, width, f.dtype, dev), _matrix(x, "x", count, width, f.dtype, dev)
    num_slots = int(state.shape[0])
    state_at = _vector(state, "state", (num_slots, width), f32, dev)
    bias_at, slots_at = _vector(bias, "bias", (width,), f32, dev), _vector(slots, "slots", (count,), i32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        if "h" not in out:
            out["h"] = torch.empty((count, width), dtype=f.dtype, device=dev)
        if slots is not None and "status" not in out:
            out["status"] = torch.empty(1, dtype=i32, device=dev)
        ldh = _matrix(out["h"], "h", count, width, f.dtype, dev)
        rc = lib.cp_recurrence_step(count, width, kind, f.data_ptr(), ldf, x.data_ptr(), ldx, bias_at, state_at, num_slots, slots_at,
                                    out["h"].data_ptr(), ldh, handle, _vector(out.get("status"), "status", (1,), i32, dev))
    if rc:
        raise CpError(rc, "cp_recurrence_step")
    if check_status and slots is not None:
        _check(out["status"], STATUS_BAD_SLOT, "a slot lies behind the last state", dev)
    return out


# ---- norms, gate and residual ----------------------------------------------------------------------


def _joint(x, y, gate, w_pre, w_post, gate_act):
    dev = _on_gpu(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x: [rows][width], not {tuple(x.shape)}")
    if gate_act not in GATES:
        raise ValueError(f"gate_act: one of {sorted(GATES)}, not {gate_act!r}")
    if y is None and (gate is not None or w_post is not None):
        raise ValueError("gate and w_post belong to y")
    return dev, int(x.shape[0]), int(x.shape[1]), GATES[gate_act]


def cp_norm_gate(x, y=None, gate=None, *, w_pre, w_post=None, gate_act="sigmoid", scale=1.0, eps=1e-6, z_dtype=None,
                 want_stats=False, out=None, stream=None):
    """r = x + scale * act(gate) * u with u = y / rms(y) * w_post (y itself without ``w_post``), and
    z = r / rms(r) * w_pre.

    ``x`` [rows][width] of the type of ``y`` and ``gate``, or float32; without ``y``, r is x and z (of ``z_dtype``, by
    default x's) its norm.  ``gate_act``: "none", "sigmoid" or "silu"; ``w_pre``, ``w_post`` [width] of one type.
    Returns a dict: ``r`` (with ``y``), ``z`` and, if wanted, ``stats`` for the backward pass."""
    import torch
    lib = load_library()
    dev, rows, width, act = _joint(x, y, gate, w_pre, w_post, gate_act)
    block = y.dtype if y is not None else z_dtype or x.dtype
    ldx = _matrix(x, "x", rows, width, x.dtype, dev)
    ldy = _matrix(y, "y", rows, width, block, dev) if y is not None else 0
    ldg = _matrix(gate, "gate", rows, width, block, dev) if gate is not None else 0
    pre_at, post_at = _vector(w_pre, "w_pre", (width,), w_pre.dtype, dev), _vector(w_post, "w_post", (width,), w_pre.dtype, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        if y is not None and "r" not in out:
            out["r"] = torch.empty((rows, width), dtype=x.dtype, device=dev)
        if "z" not in out:
            out["z"] = torch.empty((rows, width), dtype=block, device=dev)
        if want_stats and "stats" not in out:
            out["stats"] = torch.empty((2, rows), dtype=torch.float32, device=dev)
        r, z = out.get("r"), out["z"]
        ldr = _matrix(r, "r", rows, width, x.dtype, dev) if r is not None else 0
        rc = lib.cp_norm_gate(rows, width, _type(x, "x"), _type(z, "z"), _type(w_pre, "w_pre"), act, x.data_ptr(), ldx,
                              y.data_ptr() if y is not None else None, ldy, gate.data_ptr() if gate is not None else None, ldg,
                              pre_at, post_at, scale, eps, r.data_ptr() if r is not None else None, ldr, z.data_ptr(),
                              _matrix(z, "z", rows, width, block, dev),
                              _vector(out.get("stats"), "stats", (2, rows), torch.float32, dev), handle)
    if rc:
        raise CpError(rc, "cp_norm_gate")
    return out


def cp_norm_gate_backward(dr, dz, x, y=None, gate=None, *, w_pre, w_post=None, gate_act="sigmoid", scale=1.0, stats, out=None,
                          workspace=None, stream=None):
    """Gradient of cp_norm_gate for the same inputs and the ``stats`` of that call; ``dr`` may be None (0).  Returns a
    dict: ``dx``, ``dw_pre`` and, as there are such inputs, ``dy``, ``dgate``, ``dw_post``, each of its input's type."""
    import torch
    lib = load_library()
    dev, rows, width, act = _joint(x, y, gate, w_pre, w_post, gate_act)
    block = y.dtype if y is not None else dz.dtype
    ldx = _matrix(x, "x", rows, width, x.dtype, dev)
    ldy = _matrix(y, "y", rows, width, block, dev) if y is not None else 0
    ldg = _matrix(gate, "gate", rows, width, block, dev) if gate is not None else 0
    lddr = _matrix(dr, "dr", rows, width, x.dtype, dev) if dr is not None else 0
    lddz = _matrix(dz, "dz", rows, width, block, dev)
    pre_at, post_at = _vector(w_pre, "w_pre", (width,), w_pre.dtype, dev), _vector(w_post, "w_post", (width,), w_pre.dtype, dev)
    stats_at = _vector(stats, "stats", (2, rows), torch.float32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        for key, like in (("dx", x), ("dy", y), ("dgate", gate)):
            if like is not None and key not in out:
                out[key] = torch.empty((rows, width), dtype=like.dtype, device=dev)
        for key, like in (("dw_pre", w_pre), ("dw_post", w_post)):
            if like is not None and key not in out:
                out[key] = torch.empty(width, dtype=like.dtype, device=dev)
        work = _work(workspace, _need("cp_norm_gate_backward_workspace_bytes", rows, width), dev)
        at = lambda key: out[key].data_ptr() if key in out else None  # noqa: E731
        ld = lambda key, like: _matrix(out[key], key, rows, width, like.dtype, dev) if like is not None else 0  # noqa: E731
        rc = lib.cp_norm_gate_backward(rows, width, _type(x, "x"), _type(dz, "dz"), _type(w_pre, "w_pre"), act,
                                       dr.data_ptr() if dr is not None else None, lddr, dz.data_ptr(), lddz, x.data_ptr(), ldx,
                                       y.data_ptr() if y is not None else None, ldy,
                                       gate.data_ptr() if gate is not None else None, ldg, pre_at, post_at, scale, stats_at,
                                       at("dx"), ld("dx", x), at("dy"), ld("dy", y), at("dgate"), ld("dgate", gate),
                                       _vector(out["dw_pre"], "dw_pre", (width,), w_pre.dtype, dev),
                                       _vector(out.get("dw_post"), "dw_post", (width,), w_pre.dtype, dev), *_room(work), handle)
    if rc:
        raise CpError(rc, "cp_norm_gate_backward")
    return out


# ---- log probabilities of given tokens -------------------------------------------------------------

_ANY_TOKEN = 4        # the type of no tokens
_TOKEN_BYTES = {"torch.uint8": 1, "torch.int32": 4, "torch.int64": 8}


def _rows_of(logits, tokens, allow):
    import torch
    dev = _on_gpu(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits: [rows][vocab], not {tuple(logits.shape)}")
    rows, vocab = int(logits.shape[0]), int(logits.shape[1])
    ld = _matrix(logits, "logits", rows, vocab, logits.dtype, dev)
    allow_at = _vector(allow, "allow", (rows, -(-vocab // 64)), torch.int64, dev)
    if tokens is None:
        return dev, rows, vocab, ld, allow_at, (0, None, _ANY_TOKEN, 0, 0)
    size = _TOKEN_BYTES.get(str(tokens.dtype))
    if size is None:
        raise TypeError(f"tokens: uint8, int32 or int64, not {tokens.dtype}")
    if tokens.device != dev or tokens.dim() not in (1, 2) or int(tokens.shape[0]) != rows:
        raise ValueError("tokens: [rows] or [rows][given], on the device of the logits")
    given = 1 if tokens.dim() == 1 else int(tokens.shape[1])
    stride = tokens.stride()
    return dev, rows, vocab, ld, allow_at, (given, tokens.data_ptr(), size, stride[0], stride[1] if tokens.dim() == 2 else 0)


def cp_token_logprobs(logits, tokens=None, *, scale=1.0, allow=None, top=0, out=None, workspace=None, stream=None,
                      check_status=True):
    """Log probabilities of ``tokens`` under softmax(scale * logits) over the places that ``allow`` leaves.

    ``logits`` [rows][vocab]; ``tokens`` uint8, int32 or int64, [rows] or [rows][given], any strides (the
    assignments of cp_eval in vertex-major layout, or the transposed view of partition-major ones); negative ones
    are ignored.  ``allow``: bit mask, uint64-as-int64 words [rows][ceil(vocab/64)].  Returns a dict: ``logp``
    float32 as ``tokens``, ``entropy`` float32 [rows], ``stats`` for the backward pass, ``status`` and, with
    ``top`` > 0, ``top_logp`` and ``top_idx`` (int32) [rows][top].  With ``check_status`` the stream is
    synchronised and a token >= vocab raises."""
    import torch
    lib = load_library()
    dev, rows, vocab, ld, allow_at, tok = _rows_of(logits, tokens, allow)
    f32 = torch.float32
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        if tokens is not None and "logp" not in out:
            out["logp"] = torch.empty(tokens.shape, dtype=f32, device=dev)
        if "entropy" not in out:
            out["entropy"] = torch.empty(rows, dtype=f32, device=dev)
        if "stats" not in out:
            out["stats"] = torch.empty((rows, 3), dtype=f32, device=dev)
        if "status" not in out:
            out["status"] = torch.empty(1, dtype=torch.int32, device=dev)
        if top:
            if "top_logp" not in out:
                out["top_logp"] = torch.empty((rows, top), dtype=f32, device=dev)
            if "top_idx" not in out:
                out["top_idx"] = torch.empty((rows, top), dtype=torch.int32, device=dev)
        work = _work(workspace, _need("cp_token_logprobs_workspace_bytes", rows, vocab, top), dev)
        rc = lib.cp_token_logprobs(rows, vocab, _type(logits, "logits"), logits.data_ptr(), ld, scale, allow_at, *tok,
                                   _vector(out.get("logp"), "logp", tuple(tokens.shape) if tokens is not None else (), f32, dev),
                                   _vector(out["entropy"], "entropy", (rows,), f32, dev),
                                   _vector(out["stats"], "stats", (rows, 3), f32, dev), int(top),
                                   _vector(out["top_logp"], "top_logp", (rows, top), f32, dev) if top else None,
                                   _vector(out["top_idx"], "top_idx", (rows, top), torch.int32, dev) if top else None,
                                   *_room(work), handle, _vector(out["status"], "status", (1,), torch.int32, dev))
    if rc:
        raise CpError(rc, "cp_token_logprobs")
    if check_status:
        _check(out["status"], STATUS_BAD_TOKEN, "tokens holds a place >= vocab", dev)
    return out


def cp_token_logprobs_backward(logits, tokens, stats, dlogp, *, dentropy=None, scale=1.0, allow=None, out=None, stream=None,
                               check_status=True):
    """Gradient of cp_token_logprobs with respect to the logits, for the same inputs and the ``stats`` of that call.
    ``dlogp`` float32 as ``tokens`` (it may be an expanded view: one weight per partition for all rows), ``dentropy``
    float32 [rows] or None.  Returns a dict: ``dlogits`` as ``logits``.  (``check_status`` is accepted so that the
    keywords of the forward call fit; bad tokens were told there and pass nothing on here.)"""
    import torch
    lib = load_library()
    dev, rows, vocab, ld, allow_at, tok = _rows_of(logits, tokens, allow)
    stats_at = _vector(stats, "stats", (rows, 3), torch.float32, dev)
    for name, t, shape in (("dlogp", dlogp, None if tokens is None else tuple(tokens.shape)), ("dentropy", dentropy, (rows,))):
        if t is not None and (t.device != dev or t.dtype != torch.float32 or tuple(t.shape) != shape):
            raise ValueError(f"{name}: a float32 tensor of shape {shape} on the device of the logits")
    if tokens is not None and dlogp is None:
        raise ValueError("dlogp is missing")
    ds = dlogp.stride() if dlogp is not None else (0,)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        if "dlogits" not in out:
            out["dlogits"] = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
        rc = lib.cp_token_logprobs_backward(rows, vocab, _type(logits, "logits"), logits.data_ptr(), ld, scale, allow_at, *tok,
                                            stats_at, dlogp.data_ptr() if dlogp is not None else None, ds[0],
                                            ds[1] if len(ds) > 1 else 0, dentropy.data_ptr() if dentropy is not None else None,
                                            dentropy.stride(0) if dentropy is not None else 0, out["dlogits"].data_ptr(),
                                            _matrix(out["dlogits"], "dlogits", rows, vocab, logits.dtype, dev), handle)
    if rc:
        raise CpError(rc, "cp_token_logprobs_backward")
    return out
