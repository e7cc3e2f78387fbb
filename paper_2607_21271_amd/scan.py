"""Token mixing with a state of fixed size, for the blocks of an equivariant encoder: a short causal convolution along the
tokens and the selective state space scan.

Features are [B, L, C, T] (sequence, token, channel, group element).  For every sequence, channel and group element

    d_l = softplus(delta_l + delta_bias[c])
    h_l[n] = exp(d_l A[c, n]) h_{l-1}[n] + d_l Bt_l[n] x_l
    y_l = (sum_n Ct_l[n] h_l[n] + D[c] x_l) * silu(z_l)

What a channel learns (A, D, delta_bias, the convolution's weights) is shared over T, and Bt and Ct, which the tokens
choose, do not depend on the group element: both maps commute with the group action where the features that
form Bt and Ct are invariant.  One entry point each serves training (autograd), whole sequences, and few or
single tokens that carry on from a state.  This module allocates and marshals; ``eqlinear_selective_scan``,
``eqlinear_causal_conv`` and their backwards compute.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd.function import once_differentiable

from . import _lib, ops

ACTIVATIONS = {"none": _lib.EQL_ACT_NONE, "silu": _lib.EQL_ACT_SILU}


def _tokens_ready(shape, stride) -> bool:
    """Whether the elements of a token of [B, L, C, T] are contiguous."""
    return (stride[3] == 1 or shape[3] == 1) and (stride[2] == shape[3] or shape[2] == 1)


def _groups_ready(shape, stride) -> bool:
    """Whether the N of a group of [B, L, groups, N] are contiguous."""
    return stride[3] == 1 or shape[3] == 1


def _tokens(t: torch.Tensor) -> torch.Tensor:
    return t if _tokens_ready(t.shape, t.stride()) else t.contiguous()


def _groups(t: torch.Tensor) -> torch.Tensor:
    return t if _groups_ready(t.shape, t.stride()) else t.contiguous()


def _steps(shape, stride, n):
    """The first n strides, 0 for an axis of size 1."""
    return tuple(stride[i] if shape[i] > 1 else 0 for i in range(n))


def _at(t):
    return None if t is None else t.data_ptr()


def _dense(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _check_lengths(B, ref, lengths):
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (B,) or not lengths.is_contiguous()):
        raise ValueError("lengths must be a contiguous int32 [%d], got %s %s" % (B, lengths.dtype, tuple(lengths.shape)))
    ops._check_dev(ref, lengths)


def _check_out_state(name, t, shape, dtype, refs):
    """A buffer that the caller gives for the state."""
    ops._check_out(name, t, shape, dtype)
    ops._check_dev(refs[0], t)
    if torch.is_grad_enabled() and any(r is not None and r.requires_grad for r in refs + [t]):
        raise ValueError("a call that writes %s is not differentiable; use return_state" % name)
    if ops._watched():
        raise ValueError("a call that writes %s cannot be traced or transformed; use return_state" % name)


def _told(t):
    """Tells autograd of a change in place."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


# ---- selective scan -------------------------------------------------------------------------------------------------


class _ScanPlan:
    """What the calls of one problem share: the C shape (a pointer that keeps it), the bytes of workspace, states and backward
    workspace, and the shape of the states that pass.  Its calls differ in addresses only."""
    __slots__ = ("ref", "need", "states", "back", "state")

    def __init__(self, dtype, x, b, softplus, xs, ds, zs, bs, cs):
        B, L, C, T = x
        self.ref = ctypes.pointer(_lib.ScanShape(B, L, C, T, b[3], b[2], softplus, ops._DT[dtype], _steps(x, xs, 2),
                                                 _steps(x, ds, 2), (0, 0) if zs is None else _steps(x, zs, 2),
                                                 _steps(b, bs, 3), _steps(b, cs, 3)))
        self.need = _lib.eqlinear_selective_scan_workspace_bytes(self.ref)
        self.states = _lib.eqlinear_selective_scan_states_bytes(self.ref)
        self.back = _lib.eqlinear_selective_scan_backward_workspace_bytes(self.ref)
        self.state = (B, C, T, b[3])


@functools.lru_cache(maxsize=1024)
def _scan_plan(softplus, dtype, x, delta, z, A, Bt, Ct, D, delta_bias, state, types, xs, ds, zs, bs, cs):
    """Checks shapes and types; the plan of a call, None where a tensor has to be copied before it."""
    if dtype not in ops._DT:
        raise TypeError("eqlinear supports float32, float16 and bfloat16, got %s" % dtype)
    for name, t in zip(("delta", "z", "Bt", "Ct"), types):
        if t is not None and t != dtype:
            raise TypeError("%s has dtype %s, expected %s (one dtype per call)" % (name, t, dtype))
    for name, t in zip(("A", "D", "delta_bias", "state"), types[4:]):
        if t is not None and t != torch.float32:
            raise TypeError("%s must be float32, got %s" % (name, t))
    if len(x) != 4 or delta != x or (z is not None and z != x):
        raise ValueError("x, delta and z must be [B, L, C, T], got %s, %s, %s" % (tuple(x), tuple(delta), z and tuple(z)))
    B, L, C, T = x
    if C < 1 or T < 1:
        raise ValueError("x %s has no channels or no group elements" % (tuple(x),))
    if len(A) != 2 or A[0] != C or A[1] < 1:
        raise ValueError("A must be [%d, N], got %s" % (C, tuple(A)))
    if len(Bt) != 4 or Bt[:2] != x[:2] or Bt[3] != A[1] or Bt[2] < 1 or C % Bt[2] or Ct != Bt:
        raise ValueError("Bt and Ct must be [%d, %d, groups, %d] with groups that divide %d channels, got %s and %s"
                         % (B, L, A[1], C, tuple(Bt), tuple(Ct)))
    for name, s in (("D", D), ("delta_bias", delta_bias)):
        if s is not None and tuple(s) != (C,):
            raise ValueError("%s must be [%d], got %s" % (name, C, tuple(s)))
    if state is not None and tuple(state) != (B, C, T, A[1]):
        raise ValueError("state must be [%d, %d, %d, %d], got %s" % (B, C, T, A[1], tuple(state)))
    if not (_tokens_ready(x, xs) and _tokens_ready(x, ds) and (z is None or _tokens_ready(x, zs)) and _groups_ready(Bt, bs)
            and _groups_ready(Bt, cs)):
        return None
    return _ScanPlan(dtype, x, Bt, softplus, xs, ds, zs, bs, cs)


def _scan_check(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, state):
    a, b, c, d = D is None, z is None, delta_bias is None, state is None
    return _scan_plan(softplus, x.dtype, x.shape, delta.shape, None if b else z.shape, A.shape, Bt.shape, Ct.shape,
                      None if a else D.shape, None if c else delta_bias.shape, None if d else state.shape,
                      (delta.dtype, None if b else z.dtype, Bt.dtype, Ct.dtype, A.dtype, None if a else D.dtype,
                       None if c else delta_bias.dtype, None if d else state.dtype),
                      x.stride(), delta.stride(), None if b else z.stride(), Bt.stride(), Ct.stride())


def _scan_ready(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, state):
    """The tensors of a call as the kernels read them, and its plan."""
    given = (_tokens(x), _tokens(delta), A.contiguous(), _groups(Bt), _groups(Ct), None if D is None else D.contiguous(),
             None if z is None else _tokens(z), None if delta_bias is None else delta_bias.contiguous())
    state = None if state is None else state.contiguous()
    return given, state, _scan_check(*given, softplus, state)


def _scan_forward(plan, given, state, lengths, state_out, keep):
    x = given[0]
    y = _dense(x)
    ws = x.new_empty((plan.need,), dtype=torch.uint8) if plan.need else None
    states = x.new_empty((plan.states // 4,), dtype=torch.float32) if keep else None
    ops._launch("eqlinear_selective_scan", x, plan.ref, *map(_at, given), _at(lengths), _at(state), y.data_ptr(),
                _at(state_out), _at(states), _at(ws), plan.need)
    return y, states


class SelectiveScanFunction(torch.autograd.Function):
    """Autograd: the gradients of everything that is given, and of the state before the first token."""

    @staticmethod
    def forward(ctx, x, delta, A, Bt, Ct, D, z, delta_bias, state, softplus, lengths, want_state):
        ctx.set_materialize_grads(False)
        given, state, plan = _scan_ready(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, state)
        state_out = A.new_empty(plan.state) if want_state else None
        y, states = _scan_forward(plan, given, state, lengths, state_out, True)
        ctx.save_for_backward(*given, lengths, states)
        ctx.plan, ctx.has_state = plan, state is not None
        return (y, state_out) if want_state else y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gstate=None):
        *given, lengths, states = ctx.saved_tensors
        if gy is None and gstate is None:
            return (None,) * 12
        plan, x = ctx.plan, given[0]
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else gy.contiguous()
        gstate = None if gstate is None else gstate.contiguous()
        dx, ddelta, dA, dB, dC, dD, dz, dbias = grads = [None if t is None else _dense(t) for t in given]
        dstate = given[2].new_empty(plan.state) if ctx.has_state else None
        ws = x.new_empty((plan.back,), dtype=torch.uint8) if plan.back else None
        ops._launch("eqlinear_selective_scan_backward", x, plan.ref, *map(_at, given), _at(lengths), _at(states), gy.data_ptr(),
                    _at(gstate), *map(_at, (dx, ddelta, dA, dB, dC, dD, dz, dbias, dstate, ws)), plan.back)
        return (*grads, dstate, None, None, None)


def selective_scan(x: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, Bt: torch.Tensor, Ct: torch.Tensor,
                   D: torch.Tensor | None = None, z: torch.Tensor | None = None, delta_bias: torch.Tensor | None = None,
                   softplus: bool = True, lengths: torch.Tensor | None = None, state: torch.Tensor | None = None,
                   return_state: bool = False, state_out: torch.Tensor | None = None):
    """y [B, L, C, T] from x, delta and the gate z [B, L, C, T] (views whose tokens are contiguous are read as they are),
    Bt and Ct [B, L, groups, N] (channel c reads group c // (C / groups)), all of one type, and A [C, N], D and
    delta_bias [C] in float32.  ``softplus=False`` takes delta + delta_bias as the step itself.

    ``lengths`` int32 [B]: tokens of each sequence that hold data (None: L); the others give zeros and no gradient, and
    leave the state.  ``state`` float32 [B, C, T, N]: h before the first token (None: 0).  ``return_state``: (y, h after the last
    token).  ``state_out``: a buffer for that h, which may be ``state`` itself (updated in place); the call is then not
    differentiable and gives (y, state_out).

    Training keeps, until its backward pass, a float32 state before every eight tokens: 8 bytes for each element of x at 9 to 16
    states, 32 at 33 to 64, more where groups have few columns (C / groups * T is rounded up to 64 columns at 9 to 16
    states)."""
    softplus = bool(softplus)
    plan = _scan_check(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, state)
    ops._check_dev(x, delta, A, Bt, Ct, D, z, delta_bias, state)
    if lengths is not None:
        _check_lengths(x.shape[0], x, lengths)
    if state_out is not None:
        _check_out_state("state_out", state_out, (*x.shape[:1], *x.shape[2:], A.shape[1]), torch.float32,
                         [x, delta, A, Bt, Ct, D, z, delta_bias, state])
    elif not ops._no_node(*(t for t in (x, delta, A, Bt, Ct, D, z, delta_bias, state) if t is not None)):
        return SelectiveScanFunction.apply(x, delta, A, Bt, Ct, D, z, delta_bias, state, softplus, lengths,
                                           bool(return_state))
    given = (x, delta, A, Bt, Ct, D, z, delta_bias)
    if plan is None or not (A.is_contiguous() and all(t is None or t.is_contiguous() for t in (D, delta_bias, state))):
        given, state, plan = _scan_ready(*given, softplus, state)
    out = state_out
    if out is None and return_state:
        out = A.new_empty(plan.state)
    y, _ = _scan_forward(plan, given, state, lengths, out, False)
    if state_out is not None:
        _told(state_out)
    return y if out is None else (y, out)


# ---- causal convolution ---------------------------------------------------------------------------------------------


@functools.lru_cache(maxsize=1024)
def _conv_plan(act, dtype, x, weight, bias, state, types, stride):
    """Checks shapes and types; the C shape of a call (a pointer that keeps it), the bytes of its backward workspace and the
    shape of the tokens that pass."""
    if dtype not in ops._DT:
        raise TypeError("eqlinear supports float32, float16 and bfloat16, got %s" % dtype)
    for name, t in zip(("weight", "bias", "state"), types):
        if t is not None and t != dtype:
            raise TypeError("%s has dtype %s, expected %s (one dtype per call)" % (name, t, dtype))
    if len(x) != 4 or x[2] < 1 or x[3] < 1:
        raise ValueError("x must be [B, L, C, T], got %s" % (tuple(x),))
    B, L, C, T = x
    if len(weight) != 2 or weight[0] != C or weight[1] < 1:
        raise ValueError("weight must be [%d, W], got %s" % (C, tuple(weight)))
    W = weight[1]
    if bias is not None and tuple(bias) != (C,):
        raise ValueError("bias must be [%d], got %s" % (C, tuple(bias)))
    if state is not None and tuple(state) != (B, W - 1, C, T):
        raise ValueError("state must be [%d, %d, %d, %d], got %s" % (B, W - 1, C, T, tuple(state)))
    if act not in ACTIVATIONS:
        raise ValueError("activation must be one of %s, got %r" % (", ".join(ACTIVATIONS), act))
    ref = ctypes.pointer(_lib.ConvShape(B, L, C, T, W, ACTIVATIONS[act], ops._DT[dtype], 0, _steps(x, stride, 2)))
    return ref, _lib.eqlinear_causal_conv_backward_workspace_bytes(ref), (B, W - 1, C, T)


def _conv_check(x, weight, bias, act, state):
    a, b = bias is None, state is None
    return _conv_plan(act, x.dtype, x.shape, weight.shape, None if a else bias.shape, None if b else state.shape,
                      (weight.dtype, None if a else bias.dtype, None if b else state.dtype), x.stride())


def _conv_forward(plan, x, weight, bias, lengths, state, state_out):
    y = _dense(x)
    ops._launch("eqlinear_causal_conv", x, plan[0], x.data_ptr(), weight.data_ptr(), _at(bias), _at(lengths), _at(state),
                y.data_ptr(), _at(state_out))
    return y


class CausalConvFunction(torch.autograd.Function):
    """Autograd: gradients of x, weight, bias and the state before the first token."""

    @staticmethod
    def forward(ctx, x, weight, bias, state, act, lengths, want_state):
        ctx.set_materialize_grads(False)
        x = _tokens(x)
        weight, bias, state = (None if t is None else t.contiguous() for t in (weight, bias, state))
        plan = _conv_check(x, weight, bias, act, state)
        state_out = x.new_empty(plan[2]) if want_state else None
        y = _conv_forward(plan, x, weight, bias, lengths, state, state_out)
        ctx.save_for_backward(x, weight, bias, state, lengths)
        ctx.act = act
        return (y, state_out) if want_state else y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gstate=None):
        x, weight, bias, state, lengths = ctx.saved_tensors
        if gy is None and gstate is None:
            return (None,) * 7
        ref, need, _ = _conv_check(x, weight, bias, ctx.act, state)
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else gy.contiguous()
        gstate = None if gstate is None else gstate.contiguous()
        dx, dw, db, dstate = (None if t is None else _dense(t) for t in (x, weight, bias, state))
        ws = x.new_empty((need,), dtype=torch.uint8) if need else None
        ops._launch("eqlinear_causal_conv_backward", x, ref,
                    *map(_at, (x, weight, bias, lengths, state, gy, gstate, dx, dw, db, dstate, ws)), need)
        return dx, dw, db, dstate, None, None, None


def causal_conv(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none",
                lengths: torch.Tensor | None = None, state: torch.Tensor | None = None, return_state: bool = False,
                state_out: torch.Tensor | None = None):
    """y_l = act(bias[c] + sum_w weight[c, w] x_{l - W + 1 + w}) along the tokens of x [B, L, C, T] (a view whose tokens are
    contiguous is read as it is), weight [C, W], bias [C], all of one type; ``activation`` none or silu.

    ``lengths`` as in ``selective_scan``.  ``state`` [B, W - 1, C, T] of x's type: the tokens before the first (None: zeros).
    ``return_state``: (y, the last W - 1 tokens).  ``state_out``: a buffer for them, which may be ``state`` itself (updated in
    place); the call is then not differentiable and gives (y, state_out)."""
    plan = _conv_check(x, weight, bias, activation, state)
    ops._check_dev(x, weight, bias, state)
    if lengths is not None:
        _check_lengths(x.shape[0], x, lengths)
    if state_out is not None:
        _check_out_state("state_out", state_out, plan[2], x.dtype, [x, weight, bias, state])
    elif not ops._no_node(*(t for t in (x, weight, bias, state) if t is not None)):
        return CausalConvFunction.apply(x, weight, bias, state, activation, lengths, bool(return_state))
    if not _tokens_ready(x.shape, x.stride()):
        x = x.contiguous()
        plan = _conv_check(x, weight, bias, activation, state)
    weight, bias, state = weight.contiguous(), None if bias is None else bias.contiguous(), None if state is None else state.contiguous()
    out = state_out
    if out is None and return_state:
        out = x.new_empty(plan[2])
    y = _conv_forward(plan, x, weight, bias, lengths, state, out)
    if state_out is not None:
        _told(state_out)
    return y if out is None else (y, out)
