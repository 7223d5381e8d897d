"""Operators of a replayed transformer layer (include/c3_replay.h) for torch
tensors on a ROCm device.

A replay runs a layer again on every replica and votes on outputs and
gradients bit by bit, so each operator's bits depend on its inputs alone: no
atomics, sums in an order that the sizes fix.  Argument marshalling only;
every step runs in the HIP kernels of libc3.so and there is no CPU fallback.

* ``rotary(x, positions, freqs)``         rotary positions; ``inverse`` is the gradient
* ``rotary_frequencies(rot, ...)``        their frequencies, scaled for long contexts
* ``attention(q, k, v)``                  output and per-row log-sum-exp
* ``attention_grad(dout, q, k, v, out, lse)`` gradients of queries, keys and values
* ``expert_sort(ids, num_experts)``       choices sorted by expert
* ``expert_dispatch(x, order)``           tokens to their experts' rows
* ``expert_combine(y, order, weights)``   and back, weighted
* ``expert_combine_grad``, ``expert_dispatch_grad``  their gradients

The calls record no graph.  Where torch would record one, tensors that require a
gradient are refused; under ``torch.no_grad()`` and inside the forward and backward of a
``torch.autograd.Function`` they are taken.
"""
from __future__ import annotations

import ctypes
import math
import operator
import struct
from typing import NamedTuple

import torch

from . import c3
from .c3 import BF16, F16, F32, C3Error, _check, _dev_tensor, _empty, _ptr, _raw_stream, _stream

HALF, INTERLEAVED = 0, 1
MAX_HEAD_DIM = 128
MAX_EXPERTS, MAX_TOP = 512, 64
MAX_CAPTURED_SEQUENCES = 112

_CODE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_LAYOUT = {"half": HALF, "interleaved": INTERLEAVED}


class Heads(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("in_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
                ("heads", ctypes.c_int64)]


class Attention(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "dim", "causal", "window")] + [
        ("scale", ctypes.c_float), ("batch", ctypes.c_int32), ("q_tokens", ctypes.c_int64),
        ("k_tokens", ctypes.c_int64), ("packed", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("q_lens", ctypes.c_void_p), ("k_lens", ctypes.c_void_p)]


class AttnTensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride", ctypes.c_int64 * 3)]


class ExpertRows(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("top", ctypes.c_int32), ("tokens", ctypes.c_int64),
                ("hidden", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("sorted_stride", ctypes.c_int64), ("slot", ctypes.c_void_p), ("kept", ctypes.c_void_p)]


# The same fields in one step: setting them one by one costs a call several microseconds.
_HEADS = struct.Struct("@2P7q")
_POS = struct.Struct("@2q")
_ATTENTION = struct.Struct("@6ifi2q2i2P")
_ATTN_TENSOR = struct.Struct("@P3q")
_EXPERT_ROWS = struct.Struct("@2i4q2P")

_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = c3.lib()
        vp, i32, i64, sz, dbl = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t,
                                 ctypes.c_double)
        L.c3_rotary.restype = i32
        L.c3_rotary.argtypes = [vp, i32, i32, i64, i64, i64, vp, i32, vp, vp, i64, i32, i32, dbl, vp]
        for n in ("c3_attention_workspace_size", "c3_attention_grad_workspace_size"):
            getattr(L, n).restype = sz
            getattr(L, n).argtypes = [vp]
        L.c3_attention.restype = i32
        L.c3_attention.argtypes = [vp] * 7 + [sz, vp]
        L.c3_attention_grad.restype = i32
        L.c3_attention_grad.argtypes = [vp] * 11 + [sz, vp]
        L.c3_expert_sort_workspace_size.restype = sz
        L.c3_expert_sort_workspace_size.argtypes = [i64, i32]
        L.c3_expert_sort.restype = i32
        L.c3_expert_sort.argtypes = [vp, i64, i32, vp, vp, vp, vp, sz, vp]
        L.c3_expert_dispatch.restype = i32
        L.c3_expert_dispatch.argtypes = [vp] * 4
        L.c3_expert_combine.restype = i32
        L.c3_expert_combine.argtypes = [vp] * 5
        L.c3_expert_combine_grad.restype = i32
        L.c3_expert_combine_grad.argtypes = [vp] * 7
        _ready = L
    return _ready


def _no_graph(name):
    """Refuses a tensor that requires a gradient, which would stop here without a word."""
    if torch.is_grad_enabled():
        raise C3Error(f"{name} requires a gradient, which this call does not record: call it under "
                      "torch.no_grad() or in a torch.autograd.Function")


def _rows(t, name, dtype=None, device=None, dim=None):
    """A device tensor whose last dimension is contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise C3Error(f"{name} must be a tensor on a ROCm GPU device")
    if t.requires_grad:
        _no_graph(name)
    if t.dtype not in _CODE:
        raise C3Error(f"{name}: unsupported dtype {t.dtype}")
    if dtype is not None and t.dtype != dtype:
        raise C3Error(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise C3Error(f"{name} must be on {device}")
    n = t.dim()
    if dim is not None and n not in dim:
        raise C3Error(f"{name} must have {' or '.join(map(str, dim))} dimensions")
    if n and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise C3Error(f"{name}: the last dimension must be contiguous")
    return t


def _out(t, name, shape, dtype, device, stream):
    """The caller's result tensor, checked, or a new one."""
    if t is None:
        return _new(shape, dtype, device, stream)
    _rows(t, name, dtype, device)
    if t.shape != shape or any(n > 1 and s == 0 for n, s in zip(shape, t.stride())):
        raise C3Error(f"{name} must have the shape {tuple(shape)} and no repeated elements")
    return t


def _new(shape, dtype, device, stream):
    """Memory of the stream that the call runs on: memory of another one could still be in
    use there, or be given out again before the call has ended."""
    if stream is None:
        return _empty(shape, dtype, device)
    with torch.cuda.stream(stream):
        return _empty(shape, dtype, device)


def _handle(stream, device):
    """The stream's handle.  Kernels run on the current device, and the memory of another
    one is not theirs to reach."""
    at = torch.cuda.current_device()
    if device.index != at or (stream is not None and stream.device != device):
        raise C3Error(f"the tensors are on {device}: make it the current device, and pass a stream of it")
    # c3._stream would ask for the device once more, a microsecond a call
    return _raw_stream(at) if stream is None and _raw_stream is not None else _stream(stream)


def _int32(x, name):
    """A whole number that fits the call's field, which would cut it off without a word."""
    try:
        x = operator.index(x)
    except TypeError:
        raise C3Error(f"{name} must be a whole number") from None
    if not 0 <= x < 2 ** 31:
        raise C3Error(f"{name} must be in [0, 2^31)")
    return x


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, scaling: str = "none",
                       trained: int = 4096, slow: float = 1.0, fast: float = 32.0, device="cuda"):
    """Radians a position of each of the rot / 2 pairs, fp64 on the device:
    base ** (-2 i / rot), for a context ``factor`` times the ``trained`` one
    rescaled by

    * ``"linear"``: every frequency divided by the factor;
    * ``"base"``:   a base factor ** (rot / (rot - 2)) times as large, which
      divides the slowest pair by the factor and leaves the fastest;
    * ``"ramp"``:   pairs that make fewer than ``slow`` turns in the trained
      context divided, those with more than ``fast`` left, a linear ramp in
      the number of turns between."""
    if rot < 2 or rot % 2:
        raise C3Error("rot must be even and positive")
    if not base > 0 or not factor > 0:
        raise C3Error("base and factor must be positive")
    if scaling not in ("none", "linear", "base", "ramp"):
        raise C3Error(f"unknown scaling {scaling}")
    if scaling == "base":
        if rot == 2:
            raise C3Error("scaling the base needs more than one pair")
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "ramp":
        if not fast > slow:
            raise C3Error("fast must exceed slow")
        keep = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - slow) / (fast - slow))) for x in f]
        f = [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)]
    return torch.tensor(f, dtype=torch.float64, device=device)


def _strides4(t):
    """(batch, token, head) strides of [B, S, H, D] or [S, H, D]."""
    s = t.stride()
    return (s[0], s[1], s[2]) if t.dim() == 4 else (0, s[0], s[1])


def rotary(x, positions, freqs, *, layout: str = "half", inverse: bool = False,
           amplitude: float = 1.0, out=None, stream=None):
    """Rotary positions on the first 2 * len(freqs) elements of every head.

    ``x`` is a tensor [B, S, H, D] or [S, H, D], or two of them (queries and
    keys) with the same B, S and D; ``positions`` int32 or int64 [B, S] or [S].
    ``inverse`` turns back, which is the gradient.  ``out`` (same structure as
    ``x``) may be ``x`` itself.  Returns what ``out`` is, or new tensors."""
    single = isinstance(x, torch.Tensor)
    xs = (x,) if single else tuple(x)
    if len(xs) not in (1, 2):
        raise C3Error("rotary takes one tensor or two")
    first = _rows(xs[0], "x[0]", dim=(3, 4))
    shape, dtype, dev = first.shape, first.dtype, first.device
    outs = (None,) * len(xs) if out is None else (out,) if single else tuple(out)
    if len(outs) != len(xs):
        raise C3Error("out must have one tensor for each of x")
    table, done = b"", []
    for i, (t, y) in enumerate(zip(xs, outs)):
        if i:
            _rows(t, f"x[{i}]", dtype, dev, (len(shape),))
            if t.shape[:-2] != shape[:-2] or t.shape[-1] != shape[-1]:
                raise C3Error("the tensors must agree in all but their heads")
        y = _out(y, "out", t.shape, dtype, dev, stream)
        done.append(y)
        table += _HEADS.pack(t.data_ptr(), y.data_ptr(), *_strides4(t), *_strides4(y), t.shape[-2])
    B, S = shape[:2] if len(shape) == 4 else (1, shape[0])
    if not isinstance(positions, torch.Tensor) or positions.device != dev or positions.dtype not in (
            torch.int32, torch.int64):
        raise C3Error("positions must be int32 or int64 on the device of x")
    where = positions.shape
    if len(where) == 1 and where[0] == S:
        pos = _POS.pack(0, positions.stride(0))
    elif len(where) == 2 and where[0] == B and where[1] == S:
        pos = _POS.pack(*positions.stride())
    else:
        raise C3Error("positions must be [S] or [B, S]")
    _dev_tensor(freqs, "freqs")
    if freqs.requires_grad:
        _no_graph("freqs")
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or freqs.device != dev:
        raise C3Error("freqs must be fp64 [rot / 2] on the device of x")
    if layout not in _LAYOUT:
        raise C3Error(f"unknown layout {layout}")
    rc = _lib().c3_rotary(table, len(xs), _CODE[dtype], B, S, shape[-1], positions.data_ptr(),
                          positions.element_size(), pos, freqs.data_ptr(), 2 * freqs.numel(),
                          _LAYOUT[layout], int(bool(inverse)), float(amplitude), _handle(stream, dev))
    _check(rc, "c3_rotary")
    return done[0] if single else tuple(done)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _attn_tensor(t):
    return _ATTN_TENSOR.pack(t.data_ptr(), *_strides4(t))


def _attention_args(q, k, v, causal, window, scale, q_lens, k_lens):
    _rows(q, "q", dim=(3, 4))
    qs, ks = q.shape, k.shape if isinstance(k, torch.Tensor) else None
    for t, n in ((k, "k"), (v, "v")):
        _rows(t, n, q.dtype, q.device, (len(qs),))
    if ks != v.shape:
        raise C3Error("k and v must have the same shape")
    if qs[-1] != ks[-1]:
        raise C3Error("q and k must have the same head size")
    packed = len(qs) == 3
    if (q_lens is None) != (k_lens is None):
        raise C3Error("q_lens and k_lens go together")
    if not packed and qs[0] != ks[0]:
        raise C3Error("q and k must have the same batch")
    if packed and q_lens is None:
        q_lens, k_lens = [qs[0]], [ks[0]]
    batch = len(q_lens) if packed else qs[0]
    keep, at = (), (0, 0)
    if q_lens is not None:
        if len(q_lens) != batch or len(k_lens) != batch:
            raise C3Error("q_lens and k_lens need one length for each sequence")
        keep = tuple((ctypes.c_int32 * max(batch, 1))(*[_int32(n, "a length") for n in x])
                     for x in (q_lens, k_lens))
        at = tuple(ctypes.addressof(x) for x in keep)
    q_tokens, k_tokens = (qs[0], ks[0]) if packed else (qs[1], ks[1])
    try:
        a = _ATTENTION.pack(_CODE[q.dtype], qs[-2], ks[-2], qs[-1], int(bool(causal)),
                            _int32(window, "window"), (qs[-1] or 1) ** -0.5 if scale is None else scale, batch,
                            q_tokens, k_tokens, int(packed), 0, *at)
    except (struct.error, OverflowError):
        raise C3Error("scale must be a number, and sizes below 2^31") from None
    return a, keep


def _workspace(need, workspace, device, what, stream):
    if need == 0:
        raise C3Error(f"invalid {what} sizes")
    if workspace is None:
        return _new((need,), torch.uint8, device, stream)
    _dev_tensor(workspace, "workspace")
    if workspace.device != device:
        raise C3Error(f"{what} workspace must be on {device}")
    if workspace.numel() * workspace.element_size() < need:
        raise C3Error(f"{what} workspace too small")
    return workspace


def _lse(t, q, name="lse"):
    _dev_tensor(t, name)
    if t.requires_grad:
        _no_graph(name)
    if t.dtype != torch.float32 or t.shape != q.shape[:-1] or t.device != q.device:
        raise C3Error(f"{name} must be fp32 {tuple(q.shape[:-1])}")
    return t


def attention(q, k, v, *, causal: bool = False, window: int = 0, scale: float = None, q_lens=None,
              k_lens=None, out=None, lse=None, workspace=None, stream=None):
    """(out, lse) of softmax(scale q k^T) v.

    Dense: q [B, Sq, H, D], k and v [B, Sk, Hk, D], optionally with the lengths
    of each sequence (what lies behind them is padding: not looked at, zeros in
    the output).  Packed: q [sum of q_lens, H, D], k and v alike.  bf16 or fp16,
    D a multiple of 8 up to 128, H a multiple of Hk.  Lengths are host integers.
    ``causal`` lines the last query up with the last key; ``window`` > 0 leaves
    each query that many keys.  ``scale`` defaults to D ** -0.5.  lse is fp32
    [.., H]; a row that sees no key has out 0 and lse -inf.  A graph can capture the
    call and its gradient with the lengths of up to 112 sequences (more are refused
    there); the lengths are those of the capture at every replay."""
    a, keep = _attention_args(q, k, v, causal, window, scale, q_lens, k_lens)
    out = _out(out, "out", q.shape, q.dtype, q.device, stream)
    lse = _new(q.shape[:-1], torch.float32, q.device, stream) if lse is None else _lse(lse, q)
    ws = _workspace(_lib().c3_attention_workspace_size(a), workspace, q.device,
                    "attention", stream)
    rc = _lib().c3_attention(a, *map(_attn_tensor, (q, k, v, out)), _ptr(lse), _ptr(ws),
                             ws.numel() * ws.element_size(), _handle(stream, q.device))
    _check(rc, "c3_attention")
    return out, lse


def attention_grad(dout, q, k, v, out, lse, *, causal: bool = False, window: int = 0,
                   scale: float = None, q_lens=None, k_lens=None, dq=None, dk=None, dv=None,
                   workspace=None, stream=None):
    """(dq, dk, dv) of ``attention`` with the same arguments, from its ``out``
    and ``lse`` and the output's gradient."""
    a, keep = _attention_args(q, k, v, causal, window, scale, q_lens, k_lens)
    for t, n in ((dout, "dout"), (out, "out")):
        _rows(t, n, q.dtype, q.device)
        if t.shape != q.shape:
            raise C3Error(f"{n} must have the shape of q")
    _lse(lse, q)
    dq, dk, dv = (_out(t, n, x.shape, q.dtype, q.device, stream)
                  for t, x, n in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")))
    ws = _workspace(_lib().c3_attention_grad_workspace_size(a), workspace, q.device,
                    "attention_grad", stream)
    rc = _lib().c3_attention_grad(a, *map(_attn_tensor, (dout, q, k, v, out)), _ptr(lse),
                                  *map(_attn_tensor, (dq, dk, dv)), _ptr(ws), ws.numel() * ws.element_size(),
                                  _handle(stream, q.device))
    _check(rc, "c3_attention_grad")
    return dq, dk, dv


# ---------------------------------------------------------------------------
# tokens to their experts and back
# ---------------------------------------------------------------------------
class ExpertOrder(NamedTuple):
    """Choices sorted by expert (c3_expert_sort): expert e's rows are places
    offsets[e] .. offsets[e + 1] - 1; source names the choice (token * top + i)
    at each place, -1 behind the last; slot the place of each choice [T, top],
    -1 where it was dropped."""
    offsets: torch.Tensor
    source: torch.Tensor
    slot: torch.Tensor


def expert_sort(ids: torch.Tensor, num_experts: int, *, workspace=None, stream=None) -> ExpertOrder:
    """Sorts the choices ids [T, top] (int32; outside [0, num_experts): dropped)
    by expert, stably."""
    _dev_tensor(ids, "ids")
    if ids.dtype != torch.int32 or ids.dim() != 2:
        raise C3Error("ids must be int32 [tokens, top]")
    if not 1 <= ids.shape[1] <= MAX_TOP:
        raise C3Error(f"1 to {MAX_TOP} choices a token")
    num_experts = _int32(num_experts, "num_experts")
    if not 1 <= num_experts <= MAX_EXPERTS:
        raise C3Error(f"1 to {MAX_EXPERTS} experts")
    dev, n = ids.device, ids.numel()
    order = ExpertOrder(_new((num_experts + 1,), torch.int32, dev, stream),
                        _new((n,), torch.int32, dev, stream), _new(ids.shape, torch.int32, dev, stream))
    ws = _workspace(_lib().c3_expert_sort_workspace_size(n, num_experts), workspace, dev,
                    "expert_sort", stream)
    rc = _lib().c3_expert_sort(_ptr(ids), n, num_experts, _ptr(order.offsets), _ptr(order.source),
                               _ptr(order.slot), _ptr(ws), ws.numel() * ws.element_size(),
                               _handle(stream, dev))
    _check(rc, "c3_expert_sort")
    return order


def _check_order(order):
    """An order that the kernels can follow: ``ExpertOrder`` is a plain tuple, and they
    read the number of kept rows behind the last expert's first."""
    offsets, source, slot = order
    i32 = torch.int32
    try:
        dev = slot.device
        fine = (slot.is_cuda and slot.dtype == i32 and slot.dim() == 2 and slot.is_contiguous() and
                offsets.dtype == i32 and offsets.device == dev and offsets.dim() == 1 and
                offsets.numel() > 1 and offsets.is_contiguous() and
                source.dtype == i32 and source.device == dev and source.numel() == slot.numel() and
                source.dim() == 1 and source.is_contiguous())
    except AttributeError:
        fine = False
    if not fine:
        raise C3Error("the order must be that of expert_sort: int32 offsets [experts + 1], source "
                      "[tokens * top] and slot [tokens, top], contiguous and on one device")


def _expert_rows(order, token_rows, sorted_rows, dtype):
    """c3_expert_rows_t of both sides' tensors."""
    slot, offsets, dev = order.slot, order.offsets, order.slot.device
    T, top = slot.shape
    stride = []
    for t, n, rows in ((token_rows, "tokens' rows", T), (sorted_rows, "sorted rows", T * top)):
        if t.dim() != 2 or t.shape[0] != rows:
            raise C3Error(f"the {n} must be [{rows}, hidden]")
        if t.dtype != dtype or t.device != dev:
            raise C3Error("the rows must have one dtype and the order's device")
        # the stride of a single row says nothing
        stride.append(t.stride(0) if rows > 1 else max(t.shape[1], t.stride(0)))
    H = token_rows.shape[1]
    if H != sorted_rows.shape[1]:
        raise C3Error("the rows must have one hidden size")
    return stride[1], _EXPERT_ROWS.pack(_CODE[dtype], top, T, H, *stride, slot.data_ptr(),
                                        offsets.data_ptr() + 4 * (offsets.numel() - 1))


def _weights(weights, order):
    if weights is None:
        return None
    _dev_tensor(weights, "weights")
    if weights.requires_grad:
        _no_graph("weights")
    if weights.dtype != torch.float32 or (
            weights.shape != order.slot.shape or weights.device != order.slot.device):
        raise C3Error("weights must be fp32 [tokens, top] on the order's device")
    return weights


def expert_dispatch(x, order: ExpertOrder, *, out=None, stream=None):
    """Rows [T * top, hidden] sorted by expert from tokens x [T, hidden]; the
    rows behind the last kept choice are zeros."""
    _rows(x, "x", dim=(2,))
    _check_order(order)
    out = _out(out, "out", (order.slot.numel(), x.shape[1]), x.dtype, x.device, stream)
    r = _expert_rows(order, x, out, x.dtype)[1]
    _check(_lib().c3_expert_dispatch(r, _ptr(x), _ptr(out), _handle(stream, x.device)),
           "c3_expert_dispatch")
    return out


def expert_combine(y, order: ExpertOrder, weights=None, *, out=None, stream=None):
    """out[t] = sum over t's choices of weight * y[their place]; y [T * top,
    hidden], weights fp32 [T, top] or None (ones)."""
    _rows(y, "y", dim=(2,))
    _check_order(order)
    out = _out(out, "out", (order.slot.shape[0], y.shape[1]), y.dtype, y.device, stream)
    weights = _weights(weights, order)
    r = _expert_rows(order, out, y, y.dtype)[1]
    _check(_lib().c3_expert_combine(r, _ptr(y), _ptr(weights), _ptr(out),
                                    _handle(stream, y.device)), "c3_expert_combine")
    return out


def expert_combine_grad(dout, y, order: ExpertOrder, weights=None, *, dy=None, stream=None):
    """(dy [T * top, hidden], dweights fp32 [T, top]) of ``expert_combine``;
    without weights dweights is None (and y may be)."""
    _rows(dout, "dout", dim=(2,))
    _check_order(order)
    weights = _weights(weights, order)
    dy = _out(dy, "dy", (order.slot.numel(), dout.shape[1]), dout.dtype, dout.device, stream)
    sorted_stride, r = _expert_rows(order, dout, dy, dout.dtype)
    dw = None
    if weights is not None:
        _rows(y, "y", dout.dtype, dout.device, (2,))
        if y.shape != dy.shape:
            raise C3Error(f"y must be {tuple(dy.shape)}")
        if y.shape[0] > 1 and y.stride(0) != sorted_stride:
            raise C3Error("y and dy must have the same row stride")
        dw = _new(order.slot.shape, torch.float32, dout.device, stream)
    _check(_lib().c3_expert_combine_grad(r, _ptr(dout), _ptr(y if dw is not None else None),
                                         _ptr(weights), _ptr(dy), _ptr(dw), _handle(stream, dout.device)),
           "c3_expert_combine_grad")
    return dy, dw


def expert_dispatch_grad(dsorted, order: ExpertOrder, *, out=None, stream=None):
    """Gradient [T, hidden] of ``expert_dispatch``: each token's sum over its
    choices' rows of dsorted [T * top, hidden]."""
    return expert_combine(dsorted, order, None, out=out, stream=stream)
