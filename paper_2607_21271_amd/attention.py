"""Attention with a sliding window and first tokens that stay visible, for long token sequences of an encoder.

Token i of sequence b stands at position p = starts[b] + i among the lengths[b] keys of that sequence and sees key j iff

    p < lengths[b],  j < lengths[b],  j <= p + right  and  (j >= p - left or j < sinks)

(-1 is no limit).  One entry point serves training (autograd), whole sequences and single tokens over a cache: queries
may be fewer than keys, and by default are the last of them.  Query heads may share key/value heads.  This module
allocates and marshals; ``eqlinear_window_attention`` and its backward compute.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd.function import once_differentiable

from . import _lib, ops, rotary


@functools.lru_cache(maxsize=1024)
def _whole_words(shape, stride, itemsize) -> bool:
    w = 16 // itemsize
    b, token, head = _outer(shape, stride)
    return (stride[3] == 1 and b % w == 0 and token % w == 0 and head % w == 0
            and (65 * token + shape[2] * head) * itemsize < 1 << 31)


def _ready(t: torch.Tensor) -> torch.Tensor:
    """t itself where its heads start on whole 16-byte words (and a tile of its rows spans less than 2 GiB), else a
    contiguous copy."""
    if t.data_ptr() % 16 == 0 and _whole_words(t.shape, t.stride(), t.element_size()):
        return t
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)


def _dense(shape):
    return shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3], 1


def _outer(shape, stride):
    """Strides of sequence, token and head, 0 for an axis of size 1."""
    return tuple(stride[i] if shape[i] > 1 else 0 for i in range(3))


@functools.lru_cache(maxsize=1024)
def _plan(dtype, qshape, kshape, q, k, v, do, dq, dk, dv, left, right, sinks, scale):
    """The C shape of a call (a pointer that keeps it) and its workspace bytes; the strides are those of the tensors, the
    output is dense.  One problem's calls differ in addresses only."""
    o = lambda shape, stride: (0, 0, 0) if stride is None else _outer(shape, stride)
    shape = _lib.WindowShape(qshape[0], qshape[1], kshape[1], left, right, sinks, qshape[2], kshape[2], qshape[3],
                             ops._DT[dtype], scale, 0, o(qshape, q), o(kshape, k), o(kshape, v),
                             o(qshape, _dense(qshape)), o(qshape, do), o(qshape, dq), o(kshape, dk), o(kshape, dv))
    ref = ctypes.pointer(shape)
    return ref, (_lib.eqlinear_window_attention_workspace_bytes(ref) if do is None
                 else _lib.eqlinear_window_attention_backward_workspace_bytes(ref))


def _forward(q, k, v, lengths, starts, left, right, sinks, scale, want_lse):
    qshape, kshape = q.shape, k.shape
    ref, need = _plan(q.dtype, qshape, kshape, q.stride(), k.stride(), v.stride(), None, None, None, None, left, right,
                      sinks, scale)
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    # lse [B, kv_heads, Lq, heads / kv_heads]
    lse = q.new_empty(qshape[:3], dtype=torch.float32) if want_lse else None
    ws = q.new_empty((need,), dtype=torch.uint8) if need else None
    ops._launch("eqlinear_window_attention", q, ref, ops._ptr(q), ops._ptr(k), ops._ptr(v), ops._ptr(lengths),
                ops._ptr(starts), ops._ptr(o), ops._ptr(lse), ops._ptr(ws), need)
    return o, lse


def _backward(q, k, v, lengths, starts, o, lse, do, dq, dk, dv, left, right, sinks, scale):
    ref, need = _plan(q.dtype, q.shape, k.shape, q.stride(), k.stride(), v.stride(), do.stride(), dq.stride(),
                      dk.stride(), dv.stride(), left, right, sinks, scale)
    ws = q.new_empty((need,), dtype=torch.uint8) if need else None
    ops._launch("eqlinear_window_attention_backward", q, ref, ops._ptr(q), ops._ptr(k), ops._ptr(v), ops._ptr(lengths),
                ops._ptr(starts), ops._ptr(o), ops._ptr(lse), ops._ptr(do), ops._ptr(dq), ops._ptr(dk), ops._ptr(dv),
                ops._ptr(ws), need)


def _check_spans(B, dev_of, lengths, starts):
    for name, t in (("lengths", lengths), ("starts", starts)):
        if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (B,) or not t.is_contiguous()):
            raise ValueError("%s must be a contiguous int32 [%d], got %s %s" % (name, B, t.dtype, tuple(t.shape)))
    ops._check_dev(dev_of, lengths, starts)


def _check_window(left, right, sinks):
    if left < -1 or right < -1 or sinks < 0 or max(left, right, sinks) >= 1 << 63:
        raise ValueError("left and right are -1 (no limit) or at least 0, sinks at least 0; got %d, %d, %d"
                         % (left, right, sinks))


@functools.lru_cache(maxsize=1024)
def _check_shapes(q, k, v, left, right, sinks):
    if len(q) != 4 or len(k) != 4 or v != k:
        raise ValueError("q must be [B, Lq, heads, D] and k, v [B, Lk, kv_heads, D], got %s, %s, %s"
                         % (tuple(q), tuple(k), tuple(v)))
    if q[0] != k[0] or q[3] != k[3] or q[3] < 1 or k[2] < 1 or q[2] % k[2]:
        raise ValueError("q %s and k %s differ in sequences or head size, or the heads do not divide" % (tuple(q), tuple(k)))
    _check_window(left, right, sinks)


def _check(q, k, v, lengths, starts, left, right, sinks):
    ops._dtype_code(q)
    ops._check_same_dtype(q, k=k, v=v)
    _check_shapes(q.shape, k.shape, v.shape, left, right, sinks)
    ops._check_dev(q, k, v)
    if lengths is not None or starts is not None:
        _check_spans(q.shape[0], q, lengths, starts)


class WindowAttentionFunction(torch.autograd.Function):
    """Autograd: gradients of q, k and v; key/value gradients sum over the query heads that share a head."""

    @staticmethod
    def forward(ctx, q, k, v, lengths, starts, left, right, sinks, scale):
        q, k, v = _ready(q), _ready(k), _ready(v)
        o, lse = _forward(q, k, v, lengths, starts, left, right, sinks, scale, True)
        ctx.save_for_backward(q, k, v, lengths, starts, o, lse)
        ctx.args = (left, right, sinks, scale)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, go):
        q, k, v, lengths, starts, o, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
        _backward(q, k, v, lengths, starts, o, lse, _ready(go), dq, dk, dv, *ctx.args)
        return dq, dk, dv, None, None, None, None, None, None


def window_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, left: int = -1, right: int = -1, sinks: int = 0,
                     scale: float | None = None, lengths: torch.Tensor | None = None,
                     starts: torch.Tensor | None = None) -> torch.Tensor:
    """o [B, Lq, heads, D] from q [B, Lq, heads, D] and k, v [B, Lk, kv_heads, D] (views with strides are read as they
    are where heads start on 16-byte words).

    ``lengths`` int32 [B]: keys of each sequence that hold data (None: Lk).  ``starts`` int32 [B]: position of the
    first query (None: Lk - Lq, the queries are the last tokens).  A query past its sequence, or that sees no
    key, gives zeros and no gradient.  ``scale`` defaults to D ** -0.5."""
    left, right, sinks = int(left), int(right), int(sinks)
    _check(q, k, v, lengths, starts, left, right, sinks)
    scale = float(q.shape[3]) ** -0.5 if scale is None else float(scale)
    if ops._no_node(q, k, v):
        return _forward(_ready(q), _ready(k), _ready(v), lengths, starts, left, right, sinks, scale, False)[0]
    return WindowAttentionFunction.apply(q, k, v, lengths, starts, left, right, sinks, scale)


class PackedAttentionFunction(torch.autograd.Function):
    """Rotary positions and windowed attention on the packed output of one layer, qkv [B, L, heads + 2 kv_heads, D]:
    the gradient comes back in one buffer of that shape, turned back in place."""

    @staticmethod
    def forward(ctx, qkv, kv_heads, positions, freqs, sections, T, interleaved, lengths, left, right, sinks, scale):
        H = qkv.shape[2] - 2 * kv_heads
        qkv = _ready(qkv)
        qk = qkv[:, :, :H + kv_heads]
        if positions is not None:
            qk = rotary.rotary_axes(qk.detach(), positions, freqs, sections, T, interleaved)
        q, k, v = qk[:, :, :H], qk[:, :, H:], qkv[:, :, H + kv_heads:]
        starts = torch.zeros(qkv.shape[0], dtype=torch.int32, device=qkv.device) if lengths is not None else None
        o, lse = _forward(q, k, v, lengths, starts, left, right, sinks, scale, ctx.needs_input_grad[0])
        if ctx.needs_input_grad[0]:
            ctx.save_for_backward(qk, v, lengths, starts, o, lse, positions, freqs)
            ctx.args = (left, right, sinks, scale)
            ctx.turn = (sections, T, interleaved)
            ctx.heads = (H, kv_heads)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, go):
        qk, v, lengths, starts, o, lse, positions, freqs = ctx.saved_tensors
        H, kv_heads = ctx.heads
        B, L, _, D = qk.shape
        g = qk.new_empty((B, L, H + 2 * kv_heads, D))
        dqk = g[:, :, :H + kv_heads]
        _backward(qk[:, :, :H], qk[:, :, H:], v, lengths, starts, o, lse, _ready(go), dqk[:, :, :H], dqk[:, :, H:],
                  g[:, :, H + kv_heads:], *ctx.args)
        if positions is not None:
            rotary.rotary_axes_(dqk, positions, freqs, *ctx.turn, inverse=True)
        return (g,) + (None,) * 11


def packed_window_attention(qkv: torch.Tensor, kv_heads: int, positions: torch.Tensor | None = None,
                            freqs: torch.Tensor | None = None, sections=(), T: int = 1, interleaved: bool = False,
                            lengths: torch.Tensor | None = None, left: int = -1, right: int = -1, sinks: int = 0,
                            scale: float | None = None) -> torch.Tensor:
    """Self-attention on a layer's packed output qkv [B, L, heads + 2 kv_heads, D] (queries, keys, values): queries and
    keys turned by ``rotary_axes`` where positions are given, then ``window_attention`` with every token at its own
    place (tokens from lengths[b] on are padding)."""
    left, right, sinks = int(left), int(right), int(sinks)
    ops._dtype_code(qkv)
    if qkv.dim() != 4 or kv_heads < 1 or qkv.shape[3] < 1 or qkv.shape[2] <= 2 * kv_heads or (qkv.shape[2] - 2 * kv_heads) % kv_heads:
        raise ValueError("qkv must be [B, L, heads + 2 * kv_heads, D] with heads a multiple of kv_heads = %d, got %s"
                         % (kv_heads, tuple(qkv.shape)))
    _check_window(left, right, sinks)
    if positions is not None and freqs is None:
        raise ValueError("positions need freqs (rotary.axis_frequencies)")
    ops._check_dev(qkv)
    _check_spans(qkv.shape[0], qkv, lengths, None)
    if positions is not None:
        sections = tuple(int(s) for s in sections)
        rotary._check(qkv, positions, freqs, sections, T)
    scale = float(qkv.shape[3]) ** -0.5 if scale is None else float(scale)
    return PackedAttentionFunction.apply(qkv, kv_heads, positions, freqs, sections, T, interleaved, lengths, left, right,
                                         sinks, scale)
