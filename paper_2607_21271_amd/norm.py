"""Group norm with an activation over channels-last equivariant features [B, ..., C, T].

    z = (x - mean) / sqrt(var + eps) * weight[c] + bias[c],   y = act(z)

with the statistics of each sequence (image) taken over its positions, the channels of a group and the group axis T, and
one weight and bias per channel, shared over T: the map commutes with the group action, so it stands between the layers
of ``gconv``.  This module allocates and marshals; ``eqlinear_group_norm_act`` and its backward compute.
"""
from __future__ import annotations

import functools
import math

import torch
from torch.autograd.function import once_differentiable

from . import _lib, ops

ACTIVATIONS = {"none": _lib.EQL_ACT_NONE, "relu": _lib.EQL_ACT_RELU, "silu": _lib.EQL_ACT_SILU,
               "gelu": _lib.EQL_ACT_GELU}


def _ready(t: torch.Tensor) -> torch.Tensor:
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)


@functools.lru_cache(maxsize=1024)
def _check_shapes(x, weight, bias, groups, activation):
    if len(x) < 3:
        raise ValueError("x must be [B, ..., C, T], got %s" % (tuple(x),))
    C = x[-2]
    if tuple(weight) != (C,) or tuple(bias) != (C,):
        raise ValueError("weight and bias must be [%d], got %s and %s" % (C, tuple(weight), tuple(bias)))
    if groups < 1 or C % groups:
        raise ValueError("%d channels do not divide into %d groups" % (C, groups))
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be one of %s, got %r" % (", ".join(ACTIVATIONS), activation))


@functools.lru_cache(maxsize=1024)
def _plan(shape, groups, dtype):
    """(B, S, T, C, dtype code) of a call and the workspace bytes of forward and backward."""
    C, T = shape[-2:]
    S = math.prod(shape[1:-2])
    args = (shape[0], S, T, C, groups, ops._DT[dtype])
    return args, _lib.eqlinear_group_norm_act_workspace_bytes(*args), \
        _lib.eqlinear_group_norm_act_backward_workspace_bytes(*args)


def _forward(x, weight, bias, groups, act, eps, want_stats):
    (B, S, T, C, _, dt), need, _ = _plan(x.shape, groups, x.dtype)
    y = torch.empty_like(x)
    stats = x.new_empty((B, groups, 2), dtype=torch.float32) if want_stats else None
    ws = x.new_empty((need,), dtype=torch.uint8) if need else None
    ops._launch("eqlinear_group_norm_act", x, ops._ptr(x), ops._ptr(weight), ops._ptr(bias), ops._ptr(y), ops._ptr(stats),
                ops._ptr(ws), need, B, S, T, C, groups, eps, act, dt)
    return y, stats


class GroupNormActFunction(torch.autograd.Function):
    """Autograd: gradients of x, weight and bias in one call."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups, act, eps):
        x, weight, bias = _ready(x), weight.contiguous(), bias.contiguous()
        y, stats = _forward(x, weight, bias, groups, act, eps, True)
        ctx.save_for_backward(x, weight, bias, stats)
        ctx.args = (groups, act)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, weight, bias, stats = ctx.saved_tensors
        groups, act = ctx.args
        (B, S, T, C, _, dt), _, need = _plan(x.shape, groups, x.dtype)
        gy = _ready(gy)
        dx = torch.empty_like(x)
        if x.numel() == 0:
            return dx, torch.zeros_like(weight), torch.zeros_like(bias), None, None, None
        dw, db = torch.empty_like(weight), torch.empty_like(bias)
        ws = x.new_empty((need,), dtype=torch.uint8)
        ops._launch("eqlinear_group_norm_act_backward", x, ops._ptr(x), ops._ptr(weight), ops._ptr(bias),
                    ops._ptr(stats), ops._ptr(gy), ops._ptr(dx), ops._ptr(dw), ops._ptr(db), ops._ptr(ws), need, B, S, T,
                    C, groups, act, dt)
        return dx, dw, db, None, None, None


def group_norm_act(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, groups: int, activation: str = "none",
                   eps: float = 1e-5) -> torch.Tensor:
    """y of x's shape [B, ..., C, T]; weight and bias [C]; ``activation`` none, relu, silu or gelu (by erf)."""
    ops._dtype_code(x)
    ops._check_same_dtype(x, weight=weight, bias=bias)
    _check_shapes(x.shape, weight.shape, bias.shape, groups, activation)
    ops._check_dev(x, weight, bias)
    act = ACTIVATIONS[activation]
    if ops._no_node(x, weight, bias):
        return _forward(_ready(x), weight.contiguous(), bias.contiguous(), groups, act, float(eps), False)[0]
    return GroupNormActFunction.apply(x, weight, bias, groups, act, float(eps))


class GroupNormAct(torch.nn.Module):
    """Group norm with an activation: [B, ..., C, T] -> the same shape."""

    def __init__(self, C: int, groups: int, activation: str = "none", eps: float = 1e-5, device=None, dtype=None):
        super().__init__()
        self.groups, self.activation, self.eps = groups, activation, eps
        self.weight = torch.nn.Parameter(torch.ones(C, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(C, device=device, dtype=dtype))

    def forward(self, x):
        return group_norm_act(x, self.weight, self.bias, self.groups, self.activation, self.eps)
