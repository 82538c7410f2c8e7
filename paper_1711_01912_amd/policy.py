"""The operators of a learned placement policy on torch tensors (see ``include/cpeval.h``).

``cp_recurrence`` (with ``_backward`` and ``_step``), ``cp_norm_gate`` (with ``_backward``) and
``cp_token_logprobs`` (with ``_backward``) follow the C entry points of the same names.  As in
``binding``, nothing is computed here: arguments are checked, outputs and workspaces allocated, and
the library's kernels called on ``stream`` (default: the current one).  Outputs and workspaces are
allocated for that stream; inputs of another stream are the caller's to wait for and to keep (``record_stream``).
Matrices may be views whose rows are further apart than their length (slices of a fused
projection), as long as a row's elements are contiguous.  ``out`` may carry preallocated outputs
under the keys of the result, ``workspace`` a preallocated uint8 tensor.  An output lies apart from the inputs
(``CpError`` otherwise), but cp_norm_gate's and its gradient's may be an input of as wide elements, ``h`` of
cp_recurrence_step ``f`` or ``x``, and ``dlogits`` the logits of at most 256 places a row.

The submodule ``autograd`` has the same operators as differentiable functions.
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
    """The distance between the rows of a [rows][width] tensor; ``rows`` may be several axes, as long as they are equally far
    apart throughout."""
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype}, not {t.dtype}")
    shape = t.shape
    if shape[-1] != width or t.numel() != rows * width:
        raise ValueError(f"{name}: shape {tuple(shape)} does not fit {rows} rows of {width}")
    if t.is_contiguous():
        return width
    stride = t.stride()
    if width > 1 and stride[-1] != 1:
        raise ValueError(f"{name}: the elements of a row have to be contiguous (strides {tuple(stride)})")
    if rows == 1:
        return width
    ld, inner = None, 1          # rows of the axes from the last but one on that have been looked at
    for size, step in zip(shape[-2::-1], stride[-2::-1]):
        if size == 1:
            continue
        if ld is None:
            ld = step
        elif step != ld * inner:
            raise ValueError(f"{name}: all rows have to be equally far apart (strides {tuple(stride)})")
        inner *= size
    if ld < width:
        raise ValueError(f"{name}: rows overlap (strides {tuple(stride)})")
    return ld


def _vector(t, name, shape, dtype, device):
    """The address of a contiguous tensor of that shape, or None."""
    if t is None:
        return None
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype}, not {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of shape {tuple(shape)}, not {tuple(t.shape)}")
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


_HERE = contextlib.nullcontext()


def _place(device, stream):
    """What to allocate and launch under, and the stream's handle."""
    import torch
    if stream is None and device.index == torch.cuda.current_device():
        # (the handle alone: a stream object takes 3 us, as long as the launch of a step)
        return _HERE, torch._C._cuda_getCurrentRawStream(device.index)
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        raise ValueError(f"the stream is {stream.device}'s, the tensors are on {device}")
    return _other(device, stream), stream.cuda_stream


def _rows_out(out, key, like, device, dtype=None):
    """out[key], rows as `like`'s of its type or that, made if it is not there: its address and the rows' distance."""
    import torch
    t = out.get(key)
    if t is not None:
        return t.data_ptr(), _matrix(t, key, like.numel() // max(like.shape[-1], 1), like.shape[-1], dtype or like.dtype, device)
    if dtype is None and like.is_contiguous():
        t = torch.empty_like(like)
    else:
        t = torch.empty(like.shape, dtype=dtype or like.dtype, device=device)
    out[key] = t
    return t.data_ptr(), like.shape[-1]


def _vector_out(out, key, shape, dtype, device):
    """out[key], contiguous, made if it is not there: its address."""
    import torch
    t = out.get(key)
    if t is not None:
        return _vector(t, key, shape, dtype, device)
    t = out[key] = torch.empty(shape, dtype=dtype, device=device)
    return t.data_ptr()


@functools.lru_cache(maxsize=4096)
def _need(entry, *sizes):
    out = C.c_size_t(0)
    rc = getattr(load_library(), entry)(*sizes, C.byref(out))
    if rc:
        raise CpError(rc, entry)
    return int(out.value)


def _room(workspace, need, device):
    """(the workspace or a new one, which has to live until the call is made; its address and size)"""
    import torch
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace, workspace.data_ptr(), need
    if workspace.device != device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous uint8 tensor on the device of the inputs")
    return workspace, workspace.data_ptr(), workspace.numel()


def _check(status, flag, text, stream):
    if stream is not None:
        stream.synchronize()
    if int(status.item()) & flag:        # (waits for the current stream)
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
        h_at, ldh = _rows_out(out, "h", x, dev)
        last_at = _vector_out(out, "last", (count, width), f32, dev) if want_last or "last" in out else None
        carry_at = _vector_out(out, "carry", (-(-rows // RECURRENCE_CHUNK), width), f32, dev) if want_carry or "carry" in out else None
        status_at = _vector_out(out, "status", (1,), torch.int32, dev) if ptr is not None else None
        need = _need("cp_recurrence_workspace_bytes", rows, width, 0) if rows > RECURRENCE_CHUNK else 0
        work, work_at, room = _room(workspace, need, dev)
        rc = lib.cp_recurrence(rows, width, count, ptr, kind, int(bool(reverse)), f.data_ptr(), ldf, x.data_ptr(), ldx, bias_at,
                               h0_at, h_at, ldh, last_at, carry_at, work_at, room, handle, status_at)
    if rc:
        raise CpError(rc, "cp_recurrence")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to the number of rows", stream)
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
    lddh, ldf, ldx = (_matrix(dh, "dh", rows, width, f.dtype, dev), _matrix(f, "f", rows, width, f.dtype, dev),
                      _matrix(x, "x", rows, width, f.dtype, dev))
    bias_at, h0_at = _vector(bias, "bias", (width,), f32, dev), _vector(h0, "h0", (count, width), f32, dev)
    dlast_at = _vector(dlast, "dlast", (count, width), f32, dev)
    carry_at = _vector(carry, "carry", (-(-rows // RECURRENCE_CHUNK), width), f32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        df_at, lddf = _rows_out(out, "df", f, dev)
        dx_at, lddx = _rows_out(out, "dx", x, dev)
        dbias_at = _vector_out(out, "dbias", (width,), f32, dev) if bias is not None or "dbias" in out else None
        dh0_at = _vector_out(out, "dh0", (count, width), f32, dev) if h0 is not None or "dh0" in out else None
        status_at = _vector_out(out, "status", (1,), torch.int32, dev) if ptr is not None else None
        need = _need("cp_recurrence_workspace_bytes", rows, width, 1) if rows > RECURRENCE_CHUNK or dbias_at is not None else 0
        work, work_at, room = _room(workspace, need, dev)
        rc = lib.cp_recurrence_backward(rows, width, count, ptr, kind, int(bool(reverse)), dh.data_ptr(), lddh, dlast_at,
                                        f.data_ptr(), ldf, x.data_ptr(), ldx, bias_at, h0_at, carry_at, df_at, lddf, dx_at, lddx,
                                        dbias_at, dh0_at, work_at, room, handle, status_at)
    if rc:
        raise CpError(rc, "cp_recurrence_backward")
    if check_status and ptr is not None:
        _check(out["status"], STATUS_BAD_SEQUENCE, "seq_ptr does not rise from 0 to the number of rows", stream)
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
    (count, width), num_slots = f.shape, state.shape[0]
    kind, f32, i32 = _type(f, "f"), torch.float32, torch.int32
    ldf, ldx = _matrix(f, "f", count, width, f.dtype, dev), _matrix(x, "x", count, width, f.dtype, dev)
    state_at = _vector(state, "state", (num_slots, width), f32, dev)
    bias_at, slots_at = _vector(bias, "bias", (width,), f32, dev), _vector(slots, "slots", (count,), i32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        h_at, ldh = _rows_out(out, "h", x, dev)
        status_at = _vector_out(out, "status", (1,), i32, dev) if slots is not None else None
        rc = lib.cp_recurrence_step(count, width, kind, f.data_ptr(), ldf, x.data_ptr(), ldx, bias_at, state_at, num_slots, slots_at,
                                    h_at, ldh, handle, status_at)
    if rc:
        raise CpError(rc, "cp_recurrence_step")
    if check_status and slots is not None:
        _check(out["status"], STATUS_BAD_SLOT, "a slot lies behind the last state", stream)
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
    return dev, x.shape, GATES[gate_act]


def cp_norm_gate(x, y=None, gate=None, *, w_pre, w_post=None, gate_act="sigmoid", scale=1.0, eps=1e-6, z_dtype=None,
                 want_stats=False, out=None, stream=None):
    """r = x + scale * act(gate) * u with u = y / rms(y) * w_post (y itself without ``w_post``), and
    z = r / rms(r) * w_pre.

    ``x`` [rows][width] of the type of ``y`` and ``gate``, or float32; without ``y``, r is x and z (of ``z_dtype``, by
    default x's) its norm.  ``gate_act``: "none", "sigmoid" or "silu"; ``w_pre``, ``w_post`` [width] of one type.
    Returns a dict: ``r`` (with ``y``), ``z`` and, if wanted, ``stats`` for the backward pass."""
    import torch
    lib = load_library()
    dev, (rows, width), act = _joint(x, y, gate, w_pre, w_post, gate_act)
    block = y.dtype if y is not None else z_dtype or x.dtype
    ldx = _matrix(x, "x", rows, width, x.dtype, dev)
    y_at, ldy = (y.data_ptr(), _matrix(y, "y", rows, width, block, dev)) if y is not None else (None, 0)
    gate_at, ldg = (gate.data_ptr(), _matrix(gate, "gate", rows, width, block, dev)) if gate is not None else (None, 0)
    pre_at, post_at = _vector(w_pre, "w_pre", (width,), w_pre.dtype, dev), _vector(w_post, "w_post", (width,), w_pre.dtype, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        r_at, ldr = _rows_out(out, "r", x, dev) if y is not None else (None, 0)
        z_at, ldz = _rows_out(out, "z", y, dev) if y is not None else _rows_out(out, "z", x, dev, block)
        stats_at = _vector_out(out, "stats", (2, rows), torch.float32, dev) if want_stats or "stats" in out else None
        rc = lib.cp_norm_gate(rows, width, _type(x, "x"), _type(out["z"], "z"), _type(w_pre, "w_pre"), act, x.data_ptr(), ldx, y_at,
                              ldy, gate_at, ldg, pre_at, post_at, scale, eps, r_at, ldr, z_at, ldz, stats_at, handle)
    if rc:
        raise CpError(rc, "cp_norm_gate")
    return out


def cp_norm_gate_backward(dr, dz, x, y=None, gate=None, *, w_pre, w_post=None, gate_act="sigmoid", scale=1.0, stats, out=None,
                          workspace=None, stream=None):
    """Gradient of cp_norm_gate for the same inputs and the ``stats`` of that call; ``dr`` may be None (0).  Returns a
    dict: ``dx``, ``dw_pre`` and, as there are such inputs, ``dy``, ``dgate``, ``dw_post``, each of its input's type."""
    import torch
    lib = load_library()
    dev, (rows, width), act = _joint(x, y, gate, w_pre, w_post, gate_act)
    block, weight = y.dtype if y is not None else dz.dtype, w_pre.dtype
    ldx, lddz = _matrix(x, "x", rows, width, x.dtype, dev), _matrix(dz, "dz", rows, width, block, dev)
    y_at, ldy = (y.data_ptr(), _matrix(y, "y", rows, width, block, dev)) if y is not None else (None, 0)
    gate_at, ldg = (gate.data_ptr(), _matrix(gate, "gate", rows, width, block, dev)) if gate is not None else (None, 0)
    dr_at, lddr = (dr.data_ptr(), _matrix(dr, "dr", rows, width, x.dtype, dev)) if dr is not None else (None, 0)
    pre_at, post_at = _vector(w_pre, "w_pre", (width,), weight, dev), _vector(w_post, "w_post", (width,), weight, dev)
    stats_at = _vector(stats, "stats", (2, rows), torch.float32, dev)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        dx_at, lddx = _rows_out(out, "dx", x, dev)
        dy_at, lddy = _rows_out(out, "dy", y, dev) if y is not None else (None, 0)
        dg_at, lddg = _rows_out(out, "dgate", gate, dev) if gate is not None else (None, 0)
        dw_pre_at = _vector_out(out, "dw_pre", (width,), weight, dev)
        dw_post_at = _vector_out(out, "dw_post", (width,), weight, dev) if w_post is not None else None
        work, work_at, room = _room(workspace, _need("cp_norm_gate_backward_workspace_bytes", rows, width), dev)
        rc = lib.cp_norm_gate_backward(rows, width, _type(x, "x"), _type(dz, "dz"), _type(w_pre, "w_pre"), act, dr_at, lddr,
                                       dz.data_ptr(), lddz, x.data_ptr(), ldx, y_at, ldy, gate_at, ldg, pre_at, post_at, scale,
                                       stats_at, dx_at, lddx, dy_at, lddy, dg_at, lddg, dw_pre_at, dw_post_at, work_at, room, handle)
    if rc:
        raise CpError(rc, "cp_norm_gate_backward")
    return out


# ---- log probabilities of given tokens -------------------------------------------------------------

_ANY_TOKEN = 4        # the type of no tokens


@functools.lru_cache(maxsize=1)
def _token_types():
    import torch
    return {torch.uint8: 1, torch.int32: 4, torch.int64: 8}


def _rows_of(logits, tokens, allow):
    import torch
    dev = _on_gpu(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits: [rows][vocab], not {tuple(logits.shape)}")
    rows, vocab = logits.shape
    ld = _matrix(logits, "logits", rows, vocab, logits.dtype, dev)
    allow_at = _vector(allow, "allow", (rows, -(-vocab // 64)), torch.int64, dev)
    if tokens is None:
        return dev, rows, vocab, ld, allow_at, (0, None, _ANY_TOKEN, 0, 0)
    size = _token_types().get(tokens.dtype)
    if size is None:
        raise TypeError(f"tokens: uint8, int32 or int64, not {tokens.dtype}")
    shape, stride = tokens.shape, tokens.stride()
    if tokens.device != dev or len(shape) not in (1, 2) or shape[0] != rows:
        raise ValueError("tokens: [rows] or [rows][given], on the device of the logits")
    if len(shape) == 1:
        return dev, rows, vocab, ld, allow_at, (1, tokens.data_ptr(), size, stride[0], 0)
    return dev, rows, vocab, ld, allow_at, (shape[1], tokens.data_ptr(), size, *stride)


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
        logp_at = _vector_out(out, "logp", tokens.shape, f32, dev) if tokens is not None else None
        entropy_at, stats_at = _vector_out(out, "entropy", (rows,), f32, dev), _vector_out(out, "stats", (rows, 3), f32, dev)
        status_at = _vector_out(out, "status", (1,), torch.int32, dev)
        top_at, idx_at = (_vector_out(out, "top_logp", (rows, top), f32, dev),
                          _vector_out(out, "top_idx", (rows, top), torch.int32, dev)) if top else (None, None)
        work, work_at, room = _room(workspace, _need("cp_token_logprobs_workspace_bytes", rows, vocab, top), dev)
        rc = lib.cp_token_logprobs(rows, vocab, _type(logits, "logits"), logits.data_ptr(), ld, scale, allow_at, *tok, logp_at,
                                   entropy_at, stats_at, top, top_at, idx_at, work_at, room, handle, status_at)
    if rc:
        raise CpError(rc, "cp_token_logprobs")
    if check_status:
        _check(out["status"], STATUS_BAD_TOKEN, "tokens holds a place >= vocab", stream)
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
    if (dlogp is None) != (tokens is None):
        raise ValueError("dlogp belongs to tokens")
    dlogp_at, row_stride, stride, de_at, de_stride = None, 0, 0, None, 0
    if dlogp is not None:
        if dlogp.device != dev or dlogp.dtype is not torch.float32 or dlogp.shape != tokens.shape:
            raise ValueError(f"dlogp: a float32 tensor of shape {tuple(tokens.shape)} on the device of the logits")
        dlogp_at, row_stride, stride = dlogp.data_ptr(), dlogp.stride(0), dlogp.stride(1) if dlogp.dim() == 2 else 0
    if dentropy is not None:
        if dentropy.device != dev or dentropy.dtype is not torch.float32 or dentropy.shape != (rows,):
            raise ValueError(f"dentropy: a float32 tensor of shape {(rows,)} on the device of the logits")
        de_at, de_stride = dentropy.data_ptr(), dentropy.stride(0)
    out = dict(out) if out else {}
    place, handle = _place(dev, stream)
    with place:
        to, ldd = _rows_out(out, "dlogits", logits, dev)
        rc = lib.cp_token_logprobs_backward(rows, vocab, _type(logits, "logits"), logits.data_ptr(), ld, scale, allow_at, *tok,
                                            stats_at, dlogp_at, row_stride, stride, de_at, de_stride, to, ldd, handle)
    if rc:
        raise CpError(rc, "cp_token_logprobs_backward")
    return out
