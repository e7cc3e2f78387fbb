"""Norms of channels-last equivariant features [B, ..., C, T]: group norm with an activation, and the residual sum between
two norms (``residual_norm``, below).

    z = (x - mean) / sqrt(var + eps) * weight[c] + bias[c],   y = act(z)

with the statistics of each sequence (image) taken over its positions, the channels of a group and the group axis T, and
one weight and bias per channel, shared over T: the map commutes with the group action, so it stands between the layers
of ``gconv``.  This module allocates and marshals; ``eqlinear_group_norm_act`` and its backward compute.
"""
from __future__ import annotations

import ctypes
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


# ---- the residual sum between two norms -------------------------------------------------------------------------------

KINDS = {"layer": _lib.EQL_NORM_LAYER, "rms": _lib.EQL_NORM_RMS}


_RESIDUAL = ("branch", "weight", "bias", "scale", "gate", "post_weight", "post_bias")


@functools.lru_cache(maxsize=1024)
def _residual_plan(kind, eps, dtype, x, types, branch, weight, bias, scale, gate, post_weight, post_bias):
    """Checks shapes and types; the C shape of a call (a pointer that keeps it) and the bytes of its backward workspace."""
    if dtype not in ops._DT:
        raise TypeError("eqlinear supports float32, float16 and bfloat16, got %s" % dtype)
    for name, t in zip(_RESIDUAL, types):
        if t is not None and t != dtype:
            raise TypeError("%s has dtype %s, expected %s (one dtype per call)" % (name, t, dtype))
    if len(x) < 3 or x[-1] < 1 or x[-2] < 1:
        raise ValueError("x must be [B, ..., C, T], got %s" % (tuple(x),))
    if kind not in KINDS:
        raise ValueError("kind must be one of %s, got %r" % (", ".join(KINDS), kind))
    if branch is None and not (scale is gate is post_weight is None and weight is not None):
        raise ValueError("without a branch there is the norm of x alone: weight, and no scale, gate or post_weight")
    if branch is not None and branch != x:
        raise ValueError("branch must be %s, got %s" % (tuple(x), tuple(branch)))
    if (bias is not None and weight is None) or (post_bias is not None and post_weight is None):
        raise ValueError("a bias needs the weight of its norm")
    for name, s, want in (("weight", weight, x[-2:-1]), ("bias", bias, x[-2:-1]), ("scale", scale, x[-2:-1]),
                          ("gate", gate, (x[0], x[-2])), ("post_weight", post_weight, x[-2:-1]),
                          ("post_bias", post_bias, x[-2:-1])):
        if s is not None and tuple(s) != tuple(want):
            raise ValueError("%s must be %s, got %s" % (name, list(want), tuple(s)))
    ref = ctypes.pointer(_lib.ResidualShape(x[0], math.prod(x[1:-2]), x[-2], x[-1], KINDS[kind], ops._DT[dtype], eps, 0))
    return ref, _lib.eqlinear_residual_norm_backward_workspace_bytes(ref)


def _residual_check(kind, eps, x, *given):
    return _residual_plan(kind, eps, x.dtype, x.shape, tuple([None if t is None else t.dtype for t in given]),
                          *[None if t is None else t.shape for t in given])


def _residual_forward(ref, given):
    x = given[0]
    r = None if given[1] is None else torch.empty_like(x)
    h = None if given[2] is None else torch.empty_like(x)
    ops._launch("eqlinear_residual_norm", x, ref, *[None if t is None else t.data_ptr() for t in (*given, r, h)])
    return r, h


class ResidualNormFunction(torch.autograd.Function):
    """Autograd: gradients of x, the branch and every parameter; r is formed again from x and the branch."""

    @staticmethod
    def forward(ctx, x, branch, weight, bias, scale, gate, post_weight, post_bias, kind, eps):
        ctx.set_materialize_grads(False)
        given = tuple(None if t is None else t.contiguous()
                      for t in (x, branch, weight, bias, scale, gate, post_weight, post_bias))
        ctx.save_for_backward(*given)
        ctx.plan = _residual_check(kind, eps, *given)
        r, h = _residual_forward(ctx.plan[0], given)
        return h if r is None else r if h is None else (r, h)

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        given = ctx.saved_tensors
        x, branch, weight, _, scale, gate, post_weight, post_bias = given
        ref, need = ctx.plan
        if all(g is None for g in grads):
            return (None,) * 10
        gr, gh = grads if len(grads) == 2 else (None, grads[0]) if branch is None else (grads[0], None)
        gr, gh = (None if g is None else g.contiguous() for g in (gr, gh))
        out = [torch.empty_like(t) if t is not None and want else None for t, want in zip(given, ctx.needs_input_grad)]
        ws = x.new_empty((need,), dtype=torch.uint8)
        ops._launch("eqlinear_residual_norm_backward", x, ref,
                    *[None if t is None else t.data_ptr() for t in (x, branch, weight, scale, gate, post_weight, post_bias, gr, gh, *out, ws)],
                    need)
        return (*out, None, None)


def residual_norm(x: torch.Tensor, branch: torch.Tensor | None = None, weight: torch.Tensor | None = None,
                  bias: torch.Tensor | None = None, scale: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                  post_weight: torch.Tensor | None = None, post_bias: torch.Tensor | None = None, kind: str = "layer",
                  eps: float = 1e-6):
    """The end of one branch of a block and the norm before the next, on x and branch [B, ..., C, T]:

        v = norm(branch) * post_weight[c] + post_bias[c]   (branch itself without post_weight)
        r = x + scale[c] * gate[b, c] * v
        h = norm(r) * weight[c] + bias[c]

    Gives (r, h); h is None without ``weight``; without ``branch`` r is x and h its norm.  Norms go over the (C, T) of each token:
    ``kind`` layer (mean and variance) or rms.  Parameters are per channel, shared over T, of x's type; ``gate`` [B, C] is per
    sequence (a conditioned gate, or 0 and 1 / (1 - p) of a branch dropped at random).  Either result may be the one that has
    a gradient."""
    given = (x, branch, weight, bias, scale, gate, post_weight, post_bias)
    eps = float(eps)
    ref, _ = _residual_check(kind, eps, *given)
    ops._check_dev(*given)
    if ops._no_node(*[t for t in given if t is not None]):
        r, h = _residual_forward(ref, [None if t is None else t.contiguous() for t in given])
    else:
        out = ResidualNormFunction.apply(*given, kind, eps)
        r, h = (None, out) if branch is None else (out, None) if weight is None else out
    return x if branch is None else r, h
