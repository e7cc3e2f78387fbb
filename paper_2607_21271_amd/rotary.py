"""Rotary positions with several axes (time, height, width) for the heads of an equivariant encoder.

A token at positions p[a] turns channel pair c of every head by phi = p[axis(c)] * freqs[c]; the group elements of a
channel turn alike, so the map commutes with the group action (rolling the T axis).  Scores of turned queries and
keys then depend on the tokens' offsets along each axis only.  This module allocates and marshals;
``eqlinear_rotary`` computes.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd.function import once_differentiable

from . import _lib, ops


def axis_frequencies(sections, theta=10000.0, device=None) -> torch.Tensor:
    """Frequencies [sum(sections)], theta**(-i / n) for pair i of an axis of n pairs; ``theta`` a number or one per axis."""
    thetas = [float(theta)] * len(sections) if not hasattr(theta, "__len__") else [float(t) for t in theta]
    if len(thetas) != len(sections):
        raise ValueError("theta has %d values for %d axes" % (len(thetas), len(sections)))
    f = [t ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n, t in zip(sections, thetas)]
    return torch.cat(f).float().to(device)


def grid_positions(shape, prefix: int = 0, device=None) -> torch.Tensor:
    """Positions [prefix + prod(shape), len(shape)] (int32) of a grid of tokens in raster order, the first axis slowest,
    after ``prefix`` tokens (class and register tokens) at the origin, which do not turn."""
    axes = torch.meshgrid(*(torch.arange(n, dtype=torch.int32) for n in shape), indexing="ij")
    grid = torch.stack([a.reshape(-1) for a in axes], -1)
    return torch.cat((torch.zeros(prefix, len(shape), dtype=torch.int32), grid)).to(device)


@functools.lru_cache(maxsize=1024)
def _plan(dtype, shape, x, y, pos, float_pos, sections, T, interleaved, inverse):
    """The C shape of a call (a pointer that keeps it); x, y and pos are the tensors' strides."""
    B, L, N, D = shape
    outer = lambda st: tuple(st[i] if shape[i] > 1 else 0 for i in range(3))  # an axis of size 1 takes no step
    return ctypes.pointer(_lib.RotaryShape(B, L, N, D // T, T, len(sections), sections, float_pos, interleaved, inverse,
                                           ops._DT[dtype], outer(x), outer(y), pos[:2] if len(pos) == 3 else (0, pos[0])))


def _launch(x, positions, freqs, sections, T, interleaved, inverse, y):
    ref = _plan(x.dtype, x.shape, x.stride(), y.stride(), positions.stride(), positions.dtype == torch.float32, sections,
                T, interleaved, inverse)
    ops._launch("eqlinear_rotary", x, ref, ops._ptr(x), ops._ptr(positions), ops._ptr(freqs), ops._ptr(y))
    return y


def _rows(x):
    """x itself where the elements of a head are contiguous, else a contiguous copy."""
    return x if x.stride(3) == 1 or x.shape[3] == 1 else x.contiguous()


@functools.lru_cache(maxsize=1024)
def _check_shapes(x, positions, freqs, sections, T):
    if len(x) != 4:
        raise ValueError("x must be [B, L, heads, dh * T], got %s" % (tuple(x),))
    B, L, _, D = x
    if T < 1 or D % T:
        raise ValueError("head size %d is not a multiple of T = %d" % (D, T))
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) < 1 or 2 * sum(sections) > D // T:
        raise ValueError("sections %s do not fit %d channels (two to a pair, at most 4 axes)" % (sections, D // T))
    want = (L, len(sections))
    if tuple(positions) not in (want, (B,) + want):
        raise ValueError("positions must be %s or %s, got %s" % (want, (B,) + want, tuple(positions)))
    if tuple(freqs) != (sum(sections),):
        raise ValueError("freqs must be [%d], got %s" % (sum(sections), tuple(freqs)))


def _check(x, positions, freqs, sections, T):
    ops._dtype_code(x)
    _check_shapes(x.shape, positions.shape, freqs.shape, sections, T)
    if positions.dtype not in (torch.int32, torch.float32):
        raise TypeError("positions must be int32 or float32, got %s" % positions.dtype)
    if freqs.dtype != torch.float32:
        raise ValueError("freqs must be float32, got %s" % freqs.dtype)
    ops._check_dev(x, positions, freqs)


class RotaryFunction(torch.autograd.Function):
    """Autograd: the gradient of x is the inverse turn of the gradient of y; positions and frequencies get none."""

    @staticmethod
    def forward(ctx, x, positions, freqs, sections, T, interleaved, inverse):
        ctx.save_for_backward(positions, freqs)
        ctx.args = (sections, T, interleaved, inverse)
        x = _rows(x)
        return _launch(x, positions, freqs, sections, T, interleaved, inverse,
                       torch.empty_like(x, memory_format=torch.contiguous_format))

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        positions, freqs = ctx.saved_tensors
        sections, T, interleaved, inverse = ctx.args
        gy = _rows(gy)
        gx = _launch(gy, positions, freqs, sections, T, interleaved, not inverse,
                     torch.empty_like(gy, memory_format=torch.contiguous_format))
        return gx, None, None, None, None, None, None


def rotary_axes(x: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, sections, T: int = 1,
                interleaved: bool = False, inverse: bool = False) -> torch.Tensor:
    """x [B, L, heads, dh * T] with its first 2 * sum(sections) channels turned (a new tensor).

    positions [L, axes] or [B, L, axes] (int32 or float32), freqs [sum(sections)] (``axis_frequencies``); sections[a]
    pairs turn by axis a.  Pairs are channels (c, c + sum(sections)), or (2c, 2c + 1) where ``interleaved``.
    x may be a view with strides (the queries and keys of a packed buffer).  Differentiable in x."""
    sections = tuple(int(s) for s in sections)
    _check(x, positions, freqs, sections, T)
    if positions.stride(-1) != 1:
        positions = positions.contiguous()
    freqs = freqs.contiguous()
    if not ops._no_node(x):
        return RotaryFunction.apply(x, positions, freqs, sections, T, interleaved, inverse)
    x = _rows(x)
    return _launch(x, positions, freqs, sections, T, interleaved, inverse,
                   torch.empty_like(x, memory_format=torch.contiguous_format))


def rotary_axes_(x: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, sections, T: int = 1,
                 interleaved: bool = False, inverse: bool = False) -> torch.Tensor:
    """``rotary_axes`` in place, on x or on a view of it whose elements lie apart (no expanded tensor); not recorded by
    autograd, so x must not need a gradient, but a graph that saved x is told of the change."""
    sections = tuple(int(s) for s in sections)
    _check(x, positions, freqs, sections, T)
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("rotary_axes_ is not differentiable; use rotary_axes")
    if ops._watched() and (ops._is_tracing() or ops._transforms() is not None
                           or torch.autograd.forward_ad.unpack_dual(x).tangent is not None):
        raise ValueError("rotary_axes_ cannot be traced or transformed; use rotary_axes")
    if x.stride(3) != 1 and x.shape[3] != 1:
        raise ValueError("the elements of a head must be contiguous to turn in place")
    if positions.stride(-1) != 1:
        positions = positions.contiguous()
    _launch(x, positions, freqs.contiguous(), sections, T, interleaved, inverse, x)
    if not x.is_inference():
        torch.autograd.graph.increment_version(x)
    return x
