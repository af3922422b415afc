"""ctypes binding of include/dynlp_train.h: training and asking a student of propagated labels.

Arguments are torch tensors on one GPU (only their addresses are used).  Calls run on torch's current stream of that GPU, return
without waiting for it, and raise ``DynLPError`` for what the library refuses.  Outputs and scratch memory come from torch's
allocator; under HIP graph capture the calls allocate from the capture's pool and can be replayed.

Nothing here is part of torch's autograd: outputs have no history, also where inputs require gradients.  ``head_loss`` and
``embed_grad`` return the gradients, and ``adamw_step`` counts as a change of its tensors, so that a backward pass that has
saved one of them says so.
"""
from __future__ import annotations

import ctypes as ct

import numpy as np
import torch
from torch.autograd.graph import increment_version

from .binding import DynLPError, load_library

STATE_BLOCK = 256  # elements of an 8-bit state that share a scale

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INVALID = -1


class _Matrix(ct.Structure):
    _fields_ = [("data", ct.c_void_p), ("rows", ct.c_int64), ("stride", ct.c_int64), ("dim", ct.c_int32), ("type", ct.c_int32)]


class _Call(ct.Structure):
    _fields_ = [("stream", ct.c_void_p), ("workspace", ct.c_void_p), ("workspace_bytes", ct.c_int64)]


class _Tokens(ct.Structure):
    _fields_ = [("count", ct.c_int64), ("items", ct.c_int64), ("ids", ct.c_void_p), ("offsets", ct.c_void_p),
                ("weights", ct.c_void_p), ("rejected", ct.c_void_p), ("scale", ct.c_float), ("ids_are_64", ct.c_int32)]


class _Targets(ct.Structure):
    _fields_ = [("soft", ct.c_void_p), ("hard", ct.c_void_p), ("row_weight", ct.c_void_p), ("rejected", ct.c_void_p),
                ("grad_scale", ct.c_float)]


class _AdamwOptions(ct.Structure):
    _fields_ = [("lr", ct.c_double), ("beta1", ct.c_double), ("beta2", ct.c_double), ("eps", ct.c_double), ("step", ct.c_int64),
                ("grad_scale", ct.c_void_p), ("seed", ct.c_uint32), ("state_bits", ct.c_int32)]


_ADAMW_TENSOR = np.dtype([("n", "i8"), ("param", "u8"), ("grad", "u8"), ("m", "u8"), ("v", "u8"), ("m_scale", "u8"),
                          ("v_scale", "u8"), ("copy", "u8"), ("weight_decay", "f4"), ("param_type", "i4"), ("grad_type", "i4"),
                          ("copy_type", "i4")])

EXPORTS = ["dynlp_embed", "dynlp_embed_workspace", "dynlp_embed_grad", "dynlp_embed_grad_workspace", "dynlp_head_labels",
           "dynlp_head_loss", "dynlp_head_loss_workspace", "dynlp_adamw_step"]

_lib = None


def _library():
    global _lib
    if _lib is None:
        L = load_library()
        p, i32, i64 = ct.c_void_p, ct.c_int32, ct.c_int64
        m = ct.POINTER(_Matrix)
        call = ct.POINTER(_Call)
        tokens = ct.POINTER(_Tokens)
        L.dynlp_embed.argtypes = [m, tokens, m, call]
        L.dynlp_embed_grad.argtypes = [m, tokens, m, call]
        L.dynlp_head_labels.argtypes = [m, m, p, p, p, call]
        L.dynlp_head_loss.argtypes = [m, m, p, ct.POINTER(_Targets), p, m, p, p, call]
        L.dynlp_adamw_step.argtypes = [i32, p, ct.POINTER(_AdamwOptions), call]
        for name in ("dynlp_embed", "dynlp_embed_grad", "dynlp_head_labels", "dynlp_head_loss", "dynlp_adamw_step"):
            getattr(L, name).restype = ct.c_int
        L.dynlp_embed_workspace.argtypes = [i64, i64, i32]
        L.dynlp_embed_grad_workspace.argtypes = [i64, i64, i32, i64]
        L.dynlp_head_loss_workspace.argtypes = [i64, i32, i32, i32]
        for name in EXPORTS:
            if name.endswith("_workspace"):
                getattr(L, name).restype = i64
        _lib = L
    return _lib


def _refuse(message):
    raise DynLPError(_INVALID, message)


def _check(status):
    if status != 0:
        raise DynLPError(status, _lib.dynlp_last_error(None).decode())


def _matrix(t, name, device):
    """A 2-D tensor whose rows are contiguous, as dynlp_matrix."""
    if t.dim() != 2 or t.dtype not in _TYPES:
        _refuse(f"{name}: a 2-D tensor of float32, bfloat16 or float16 is wanted")
    if t.device != device:
        _refuse(f"{name} is on {t.device}, not on {device}")
    rows, dim = t.shape
    stride, step = t.stride()
    if rows and dim > 1 and step != 1:  # without rows strides say nothing, and are zeros where numpy made the tensor
        _refuse(f"{name}: the elements of a row have to be contiguous")
    return _Matrix(t.data_ptr(), rows, stride if rows > 1 else max(dim, 1), dim, _TYPES[t.dtype])


def _vector(t, name, dtype, count, device):
    """Address of a contiguous tensor of `count` elements (None: 0)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != count or not t.is_contiguous():
        _refuse(f"{name}: a contiguous tensor of {count} elements of {dtype} is wanted")
    if t.device != device:
        _refuse(f"{name} is on {t.device}, not on {device}")
    return t.data_ptr()


def _device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name}: a tensor on the GPU is wanted")
    return t.device


# The handle of the current stream without making a Stream object of it (1.8 us less per call), where torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _run(device, function, *args):
    """function(*args) with the tensors' GPU as the current one."""
    if torch.cuda.current_device() == device.index:
        return function(*args)
    with torch.cuda.device(device):
        return function(*args)


def _call(device, nbytes=0):
    """(dynlp_call on the current stream, what has to live until the call has been made)."""
    if not nbytes:
        return _Call(_raw_stream(device.index), None, 0), None
    space = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return _Call(_raw_stream(device.index), space.data_ptr(), nbytes), space


def _tokens(ids, offsets, weights, scale, rejected, device):
    if ids.dim() != 1 or ids.dtype not in (torch.int32, torch.int64):
        _refuse("ids: a 1-D tensor of int32 or int64 is wanted")
    count = ids.numel()
    items = count
    if offsets is not None:
        items = offsets.numel() - 1
        if offsets.dim() != 1 or items < 0:
            _refuse("offsets: a 1-D tensor of one element more than there are items is wanted")
    return _Tokens(count, items, _vector(ids, "ids", ids.dtype, count, device),
                   _vector(offsets, "offsets", torch.int64, items + 1, device),
                   _vector(weights, "weights", torch.float32, count, device),
                   _vector(rejected, "rejected", torch.int32, 1, device), float(scale), ids.dtype == torch.int64)


def embed(table, ids, offsets=None, weights=None, scale=1.0, *, rejected=None):
    """dynlp_embed.  table [V, D]; ids [T] int32 or int64 (negative: padding); offsets [B + 1] int64, or None for one row per token;
    weights [T] float32 or None.  Returns [B, D] of the table's type.  rejected: an int32 tensor of one element that grows by the
    number of ids that are not below V, or None."""
    device = _device(table, "table")
    L = _library()
    t = _tokens(ids, offsets, weights, scale, rejected, device)
    m = _matrix(table, "table", device)
    out = table.new_empty((t.items, m.dim))
    call, space = _call(device, L.dynlp_embed_workspace(t.count, t.items, m.dim) if offsets is not None else 0)
    to = _Matrix(out.data_ptr(), t.items, max(m.dim, 1), m.dim, m.type)
    _check(_run(device, L.dynlp_embed, m, t, to, call))
    return out


def embed_grad(grad, ids, num_rows, offsets=None, weights=None, scale=1.0, *, dtype=torch.float32, rejected=None):
    """dynlp_embed_grad.  grad [B, D]: gradient of what ``embed`` returned for the same tokens.  Returns the table's gradient
    [num_rows, D] of ``dtype`` (float32, or grad's type)."""
    device = _device(grad, "grad")
    L = _library()
    t = _tokens(ids, offsets, weights, scale, rejected, device)
    m = _matrix(grad, "grad", device)
    if dtype not in _TYPES:
        _refuse("dtype: float32, bfloat16 or float16 is wanted")
    if num_rows < 0:
        _refuse(f"{num_rows} rows")
    out = grad.new_empty((num_rows, m.dim), dtype=dtype)
    call, space = _call(device, L.dynlp_embed_grad_workspace(t.count, t.items, m.dim, num_rows))
    to = _Matrix(out.data_ptr(), num_rows, max(m.dim, 1), m.dim, _TYPES[dtype])
    _check(_run(device, L.dynlp_embed_grad, m, t, to, call))
    return out


def head_labels(h, weight, bias=None, soft=True, hard=True):
    """dynlp_head_labels.  h [N, D], weight [C, D] of h's type, bias [C] float32 or None.  Returns (soft [N, C] float32 or None,
    hard [N] int32 or None), like ``DynLP.get_labels``."""
    device = _device(h, "h")
    L = _library()
    m, w = _matrix(h, "h", device), _matrix(weight, "weight", device)
    b = _vector(bias, "bias", torch.float32, w.rows, device)
    so = h.new_empty((m.rows, w.rows), dtype=torch.float32) if soft else None
    ho = h.new_empty(m.rows, dtype=torch.int32) if hard else None
    call, _ = _call(device)
    _check(_run(device, L.dynlp_head_labels, m, w, b, so.data_ptr() if soft else None, ho.data_ptr() if hard else None, call))
    return so, ho


def head_loss(h, weight, bias, target, *, row_weight=None, grad_scale=1.0, grads=True, rejected=None):
    """dynlp_head_loss.  target: soft rows [N, C] float32 (what ``DynLP.get_labels`` returns first), or classes [N] int32 (what it
    returns second; negative: the row is left out); row_weight [N] float32 or None.  Returns (loss [N] float32, dh [N, D] of h's type,
    dweight [C, D] float32, dbias [C] float32); the last three are None with grads=False."""
    device = _device(h, "h")
    L = _library()
    m, w = _matrix(h, "h", device), _matrix(weight, "weight", device)
    b = _vector(bias, "bias", torch.float32, w.rows, device)
    if target.dim() == 2 and tuple(target.shape) != (m.rows, w.rows):
        _refuse(f"target: {m.rows} rows of {w.rows} classes are wanted")
    soft = target.dim() == 2
    y = _vector(target, "target", torch.float32 if soft else torch.int32, m.rows * w.rows if soft else m.rows, device)
    t = _Targets(y if soft else None, None if soft else y, _vector(row_weight, "row_weight", torch.float32, m.rows, device),
                 _vector(rejected, "rejected", torch.int32, 1, device), float(grad_scale))
    loss = h.new_empty(m.rows, dtype=torch.float32)
    if not grads:
        call, _ = _call(device)
        _check(_run(device, L.dynlp_head_loss, m, w, b, t, loss.data_ptr(), None, None, None, call))
        return loss, None, None, None
    dh = h.new_empty((m.rows, m.dim))
    dweight = h.new_empty((w.rows, m.dim), dtype=torch.float32)
    dbias = h.new_empty(w.rows, dtype=torch.float32)
    call, space = _call(device, L.dynlp_head_loss_workspace(m.rows, m.dim, w.rows, m.type))
    to = _Matrix(dh.data_ptr(), m.rows, max(m.dim, 1), m.dim, m.type)
    _check(_run(device, L.dynlp_head_loss, m, w, b, t, loss.data_ptr(), to, dweight.data_ptr(), dbias.data_ptr(), call))
    return loss, dh, dweight, dbias


def adamw_state(param, bits=32):
    """Zero states of a tensor for ``adamw_step``: (m, v) float32, or with bits=8 (m, r float8_e4m3fn, their scales float32)."""
    n = param.numel()
    if bits == 32:
        return tuple(torch.zeros(n, dtype=torch.float32, device=param.device) for _ in range(2))
    if bits != 8:
        _refuse(f"states of {bits} bits: 32 or 8 are possible")
    codes = tuple(torch.zeros(n, dtype=torch.uint8, device=param.device).view(torch.float8_e4m3fn) for _ in range(2))
    return codes + tuple(torch.zeros(-(-n // STATE_BLOCK), dtype=torch.float32, device=param.device) for _ in range(2))


def adamw_step(params, grads, states, *, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, copies=None, grad_scale=None,
               seed=0):
    """dynlp_adamw_step on lists of tensors: params and states (see ``adamw_state``) are updated in place, copies (or None) receive the
    new parameters in their own type.  weight_decay: one number, or one for each tensor.  step: 1 for the first.  grad_scale: a
    float32 tensor of one element on the GPU that all gradients are multiplied by, or None.  seed: of the 8-bit states' rounding."""
    params, grads, states = list(params), list(grads), list(states)
    count = len(params)
    if len(grads) != count or len(states) != count or (copies is not None and len(copies) != count):
        _refuse(f"{count} tensors, {len(grads)} gradients, {len(states)} states")
    if count == 0:
        return
    device = _device(params[0], "params[0]")
    bits8 = len(states[0]) == 4
    table = np.zeros(count, dtype=_ADAMW_TENSOR)
    n = [p.numel() for p in params]
    columns = {"param": params, "grad": grads, "m": [s[0] for s in states], "v": [s[1] for s in states]}
    if any(len(s) != (4 if bits8 else 2) for s in states):
        _refuse("states: all in 32 bits (two tensors each) or all in 8 (four)")
    if copies is not None:
        columns["copy"] = copies
    here = [device.index] * count
    for name, tensors in columns.items():
        if ([t.numel() for t in tensors] != n or [t.get_device() for t in tensors] != here
                or not all([t.is_contiguous() for t in tensors])):
            _refuse(f"{name}: a contiguous tensor on {device}, of as many elements as its parameter, is wanted for each")
        table[name] = [t.data_ptr() for t in tensors]
        types = [t.dtype for t in tensors]
        if name in ("param", "grad", "copy"):
            kinds = [_TYPES.get(t, -1) for t in types]
            if min(kinds) < 0:
                _refuse(f"{name}: tensors of float32, bfloat16 or float16 are wanted")
            table[name + "_type"] = kinds
        elif types != [torch.float8_e4m3fn if bits8 else torch.float32] * count:
            _refuse("states: tensors of float8_e4m3fn and their scales, or of float32, are wanted")
    if bits8:
        for name, at in (("m_scale", 2), ("v_scale", 3)):
            table[name] = [_vector(s[at], name, torch.float32, -(-n[k] // STATE_BLOCK), device) for k, s in enumerate(states)]
    table["n"] = n
    if isinstance(weight_decay, (list, tuple)) and len(weight_decay) != count:
        _refuse(f"{len(weight_decay)} weight decays for {count} tensors")
    table["weight_decay"] = weight_decay
    o = _AdamwOptions(lr, betas[0], betas[1], eps, step, _vector(grad_scale, "grad_scale", torch.float32, 1, device),
                      seed & 0xFFFFFFFF, 8 if bits8 else 32)
    L = _library()
    call, _ = _call(device)
    _check(_run(device, L.dynlp_adamw_step, count, table.ctypes.data, o, call))
    # what autograd has saved of these tensors is no longer theirs
    increment_version([*params, *(t for s in states for t in s), *(copies or ())])
