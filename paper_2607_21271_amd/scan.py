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


def _tokens(t: torch.Tensor) -> torch.Tensor:
    """t [B, L, C, T] itself where the elements of a token are contiguous and no stride is negative (none is), else a
    contiguous copy."""
    C, T = t.shape[2:]
    st = t.stride()
    return t if (st[3] == 1 or T == 1) and (st[2] == T or C == 1) else t.contiguous()


def _groups(t: torch.Tensor) -> torch.Tensor:
    """t [B, L, groups, N] itself where the N of a group are contiguous, else a contiguous copy."""
    return t if t.stride(3) == 1 or t.shape[3] == 1 else t.contiguous()


def _steps(shape, stride, n):
    """The first n strides, 0 for an axis of size 1."""
    return tuple(stride[i] if shape[i] > 1 else 0 for i in range(n))


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


@functools.lru_cache(maxsize=1024)
def _scan_plan(dtype, shape, bshape, softplus, x, delta, z, b, c):
    """The C shape of a call (a pointer that keeps it), and the bytes of its workspace, states and backward workspace."""
    B, L, C, T = shape
    ref = ctypes.pointer(_lib.ScanShape(B, L, C, T, bshape[3], bshape[2], softplus, ops._DT[dtype], _steps(shape, x, 2),
                                        _steps(shape, delta, 2), (0, 0) if z is None else _steps(shape, z, 2),
                                        _steps(bshape, b, 3), _steps(bshape, c, 3)))
    return (ref, _lib.eqlinear_selective_scan_workspace_bytes(ref), _lib.eqlinear_selective_scan_states_bytes(ref),
            _lib.eqlinear_selective_scan_backward_workspace_bytes(ref))


def _scan_call(x, delta, Bt, Ct, z, softplus):
    return _scan_plan(x.dtype, x.shape, Bt.shape, softplus, x.stride(), delta.stride(), None if z is None else z.stride(),
                      Bt.stride(), Ct.stride())


def _scan_forward(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, lengths, state, state_out, keep):
    ref, need, states_bytes, _ = _scan_call(x, delta, Bt, Ct, z, softplus)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    ws = x.new_empty((need,), dtype=torch.uint8) if need else None
    states = x.new_empty((states_bytes // 4,), dtype=torch.float32) if keep else None
    p = ops._ptr
    ops._launch("eqlinear_selective_scan", x, ref, p(x), p(delta), p(A), p(Bt), p(Ct), p(D), p(z), p(delta_bias), p(lengths),
                p(state), p(y), p(state_out), p(states), p(ws), need)
    return y, states


class SelectiveScanFunction(torch.autograd.Function):
    """Autograd: the gradients of everything that is given, and of the state before the first token."""

    @staticmethod
    def forward(ctx, x, delta, A, Bt, Ct, D, z, delta_bias, state, softplus, lengths, want_state):
        ctx.set_materialize_grads(False)
        x, delta, Bt, Ct = _tokens(x), _tokens(delta), _groups(Bt), _groups(Ct)
        z = None if z is None else _tokens(z)
        A, D, delta_bias, state = (None if t is None else t.contiguous() for t in (A, D, delta_bias, state))
        B, _, C, T = x.shape
        state_out = A.new_empty((B, C, T, A.shape[1])) if want_state else None
        y, states = _scan_forward(x, delta, A, Bt, Ct, D, z, delta_bias, softplus, lengths, state, state_out, True)
        ctx.save_for_backward(x, delta, A, Bt, Ct, D, z, delta_bias, lengths, states)
        ctx.args = (softplus, state is not None)
        return (y, state_out) if want_state else y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gstate=None):
        x, delta, A, Bt, Ct, D, z, delta_bias, lengths, states = ctx.saved_tensors
        softplus, has_state = ctx.args
        if gy is None and gstate is None:
            return (None,) * 12
        ref, _, _, need = _scan_call(x, delta, Bt, Ct, z, softplus)
        new = lambda t: None if t is None else torch.empty_like(t, memory_format=torch.contiguous_format)
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else gy.contiguous()
        gstate = None if gstate is None else gstate.contiguous()
        dx, ddelta, dA, dB, dC, dD, dz, dbias = (new(t) for t in (x, delta, A, Bt, Ct, D, z, delta_bias))
        B, _, C, T = x.shape
        dstate = A.new_empty((B, C, T, A.shape[1])) if has_state else None
        ws = x.new_empty((need,), dtype=torch.uint8) if need else None
        p = ops._ptr
        ops._launch("eqlinear_selective_scan_backward", x, ref, p(x), p(delta), p(A), p(Bt), p(Ct), p(D), p(z), p(delta_bias),
                    p(lengths), p(states), p(gy), p(gstate), p(dx), p(ddelta), p(dA), p(dB), p(dC), p(dD), p(dz), p(dbias),
                    p(dstate), p(ws), need)
        return dx, ddelta, dA, dB, dC, dD, dz, dbias, dstate, None, None, None


@functools.lru_cache(maxsize=1024)
def _check_scan_shapes(x, delta, z, A, Bt, Ct, D, delta_bias, state):
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
    differentiable and gives (y, state_out)."""
    ops._dtype_code(x)
    ops._check_same_dtype(x, delta=delta, z=z, Bt=Bt, Ct=Ct)
    for name, t in (("A", A), ("D", D), ("delta_bias", delta_bias), ("state", state)):
        if t is not None and t.dtype != torch.float32:
            raise TypeError("%s must be float32, got %s" % (name, t.dtype))
    shape = lambda t: None if t is None else t.shape
    _check_scan_shapes(x.shape, delta.shape, shape(z), A.shape, Bt.shape, Ct.shape, shape(D), shape(delta_bias), shape(state))
    ops._check_dev(x, delta, A, Bt, Ct, D, z, delta_bias, state)
    if lengths is not None:
        _check_lengths(x.shape[0], x, lengths)
    softplus = bool(softplus)
    given = [x, delta, A, Bt, Ct, D, z, delta_bias, state]
    B, _, C, T = x.shape
    if state_out is not None:
        _check_out_state("state_out", state_out, (B, C, T, A.shape[1]), torch.float32, given)
    elif not ops._no_node(*(t for t in given if t is not None)):
        return SelectiveScanFunction.apply(x, delta, A, Bt, Ct, D, z, delta_bias, state, softplus, lengths,
                                           bool(return_state))
    out = state_out
    if out is None and return_state:
        out = A.new_empty((B, C, T, A.shape[1]))
    A, D, delta_bias, state = (None if t is None else t.contiguous() for t in (A, D, delta_bias, state))
    y, _ = _scan_forward(_tokens(x), _tokens(delta), A, _groups(Bt), _groups(Ct), D, None if z is None else _tokens(z),
                         delta_bias, softplus, lengths, state, out, False)
    if state_out is not None:
        _told(state_out)
    return y if out is None else (y, out)


# ---- causal convolution ---------------------------------------------------------------------------------------------


@functools.lru_cache(maxsize=1024)
def _conv_plan(dtype, shape, W, act, x):
    """The C shape of a call (a pointer that keeps it) and the bytes of its backward workspace."""
    B, L, C, T = shape
    ref = ctypes.pointer(_lib.ConvShape(B, L, C, T, W, act, ops._DT[dtype], 0, _steps(shape, x, 2)))
    return ref, _lib.eqlinear_causal_conv_backward_workspace_bytes(ref)


def _conv_forward(x, weight, bias, act, lengths, state, state_out):
    ref, _ = _conv_plan(x.dtype, x.shape, weight.shape[1], act, x.stride())
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    p = ops._ptr
    ops._launch("eqlinear_causal_conv", x, ref, p(x), p(weight), p(bias), p(lengths), p(state), p(y), p(state_out))
    return y


class CausalConvFunction(torch.autograd.Function):
    """Autograd: gradients of x, weight, bias and the state before the first token."""

    @staticmethod
    def forward(ctx, x, weight, bias, state, act, lengths, want_state):
        ctx.set_materialize_grads(False)
        x = _tokens(x)
        weight, bias, state = (None if t is None else t.contiguous() for t in (weight, bias, state))
        B, _, C, T = x.shape
        state_out = x.new_empty((B, weight.shape[1] - 1, C, T)) if want_state else None
        y = _conv_forward(x, weight, bias, act, lengths, state, state_out)
        ctx.save_for_backward(x, weight, bias, state, lengths)
        ctx.act = act
        return (y, state_out) if want_state else y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gstate=None):
        x, weight, bias, state, lengths = ctx.saved_tensors
        if gy is None and gstate is None:
            return (None,) * 7
        ref, need = _conv_plan(x.dtype, x.shape, weight.shape[1], ctx.act, x.stride())
        new = lambda t: None if t is None else torch.empty_like(t, memory_format=torch.contiguous_format)
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else gy.contiguous()
        gstate = None if gstate is None else gstate.contiguous()
        dx, dw, db, dstate = (new(t) for t in (x, weight, bias, state))
        ws = x.new_empty((need,), dtype=torch.uint8) if need else None
        p = ops._ptr
        ops._launch("eqlinear_causal_conv_backward", x, ref, p(x), p(weight), p(bias), p(lengths), p(state), p(gy), p(gstate),
                    p(dx), p(dw), p(db), p(dstate), p(ws), need)
        return dx, dw, db, dstate, None, None, None


@functools.lru_cache(maxsize=1024)
def _check_conv_shapes(x, weight, bias, state, activation):
    if len(x) != 4 or x[2] < 1 or x[3] < 1:
        raise ValueError("x must be [B, L, C, T], got %s" % (tuple(x),))
    B, _, C, T = x
    if len(weight) != 2 or weight[0] != C or weight[1] < 1:
        raise ValueError("weight must be [%d, W], got %s" % (C, tuple(weight)))
    if bias is not None and tuple(bias) != (C,):
        raise ValueError("bias must be [%d], got %s" % (C, tuple(bias)))
    if state is not None and tuple(state) != (B, weight[1] - 1, C, T):
        raise ValueError("state must be [%d, %d, %d, %d], got %s" % (B, weight[1] - 1, C, T, tuple(state)))
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be one of %s, got %r" % (", ".join(ACTIVATIONS), activation))


def causal_conv(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none",
                lengths: torch.Tensor | None = None, state: torch.Tensor | None = None, return_state: bool = False,
                state_out: torch.Tensor | None = None):
    """y_l = act(bias[c] + sum_w weight[c, w] x_{l - W + 1 + w}) along the tokens of x [B, L, C, T] (a view whose tokens are
    contiguous is read as it is), weight [C, W], bias [C], all of one type; ``activation`` none or silu.

    ``lengths`` as in ``selective_scan``.  ``state`` [B, W - 1, C, T] of x's type: the tokens before the first (None: zeros).
    ``return_state``: (y, the last W - 1 tokens).  ``state_out``: a buffer for them, which may be ``state`` itself (updated in
    place); the call is then not differentiable and gives (y, state_out)."""
    ops._dtype_code(x)
    ops._check_same_dtype(x, weight=weight, bias=bias, state=state)
    shape = lambda t: None if t is None else t.shape
    _check_conv_shapes(x.shape, weight.shape, shape(bias), shape(state), activation)
    ops._check_dev(x, weight, bias, state)
    if lengths is not None:
        _check_lengths(x.shape[0], x, lengths)
    act = ACTIVATIONS[activation]
    given = [x, weight, bias, state]
    B, _, C, T = x.shape
    if state_out is not None:
        _check_out_state("state_out", state_out, (B, weight.shape[1] - 1, C, T), x.dtype, given)
    elif not ops._no_node(*(t for t in given if t is not None)):
        return CausalConvFunction.apply(x, weight, bias, state, act, lengths, bool(return_state))
    out = state_out
    if out is None and return_state:
        out = x.new_empty((B, weight.shape[1] - 1, C, T))
    y = _conv_forward(_tokens(x), weight.contiguous(), None if bias is None else bias.contiguous(), act, lengths,
                      None if state is None else state.contiguous(), out)
    if state_out is not None:
        _told(state_out)
    return y if out is None else (y, out)
