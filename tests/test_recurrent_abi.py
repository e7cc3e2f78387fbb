"""Argument checks of the recurrent operators' C entry points, which come before any HIP call, and their size queries
(CPU)."""
import ctypes
import os
import re

import pytest

from paper_2607_21271_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, STEP = 1 << 40, 1 << 34  # never dereferenced
INV, UNS, ALI, WS, DEV = (L.EQL_ERR_INVALID_ARG, L.EQL_ERR_UNSUPPORTED, L.EQL_ERR_ALIGNMENT, L.EQL_ERR_WORKSPACE,
                          L.EQL_ERR_NO_DEVICE)
needs_no_gpu = pytest.mark.skipif(__import__("torch").cuda.device_count() > 0, reason="addresses that hold nothing")


def test_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "eqlinear_recurrent.h")).read()
    names = sorted(set(re.findall(r"\b(eqlinear_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert len(names) == 11
    for n in names:
        assert hasattr(L.lib(), n) and n in L.SIGNATURES and callable(getattr(L, n)), n


# ---- selective scan ----

def scan_shape(B=2, L_=300, C=12, T=4, N=16, G=2, softplus=1, dt=L.EQL_F16, xs=None, bs=None):
    xs = xs or (C * T * L_, C * T)
    bs = bs or (L_ * G * N, G * N, N)
    return L.ScanShape(B, L_, C, T, N, G, softplus, dt, xs, xs, xs, bs, bs)


SCAN_IN = ("x", "delta", "A", "b", "c", "D", "z", "bias", "lengths", "state_in")


def scan(shape=True, back=False, need=None, **kw):
    at = {n: P + i * STEP for i, n in enumerate(SCAN_IN + ("y", "state_out", "states", "dy", "d_state_out", "dx", "ddelta", "dA",
                                                           "db", "dc", "dD", "dz", "dbias", "d_state_in", "ws"))}
    size = {k: kw.pop(k) for k in list(kw) if k in scan_shape.__code__.co_varnames}
    at.update(kw)
    s = scan_shape(**size)
    ref = ctypes.byref(s) if shape else None
    g = lambda *n: [at[k] for k in n]
    if back:
        nws = L.eqlinear_selective_scan_backward_workspace_bytes(ref) if need is None else need
        return L.eqlinear_selective_scan_backward(ref, *g("x", "delta", "A", "b", "c", "D", "z", "bias", "lengths", "states", "dy",
                                                          "d_state_out", "dx", "ddelta", "dA", "db", "dc", "dD", "dz", "dbias",
                                                          "d_state_in", "ws"), nws, None)
    nws = L.eqlinear_selective_scan_workspace_bytes(ref) if need is None else need
    return L.eqlinear_selective_scan(ref, *g("x", "delta", "A", "b", "c", "D", "z", "bias", "lengths", "state_in", "y", "state_out",
                                             "states", "ws"), nws, None)


SCAN_BAD = [
    (dict(shape=False), INV), (dict(dt=3), INV), (dict(B=-1), INV), (dict(L_=-1), INV), (dict(C=0), INV), (dict(N=0), INV),
    (dict(G=5), INV), (dict(G=0), INV), (dict(softplus=2), INV), (dict(T=17), UNS), (dict(N=65), UNS), (dict(C=65536, T=2), UNS),
    (dict(B=(1 << 20) + 1), UNS), (dict(L_=(1 << 30) + 1), UNS), (dict(B=1 << 20, L_=1 << 30), UNS),
    (dict(x=None), INV), (dict(delta=None), INV), (dict(A=None), INV), (dict(b=None), INV), (dict(c=None), INV),
    (dict(xs=(-1, 48)), INV), (dict(xs=(300 * 48, -48)), INV), (dict(xs=(1 << 46, 48)), INV), (dict(bs=(9600, 32, -16)), INV),
    (dict(x=P + 1), ALI), (dict(A=P + 2 * STEP + 2), ALI), (dict(lengths=P + 8 * STEP + 2), ALI), (dict(z=P + 6 * STEP + 1), ALI)]


@pytest.mark.parametrize("kw,status", SCAN_BAD)
@pytest.mark.parametrize("back", [False, True])
def test_scan_arguments(kw, status, back):
    assert scan(back=back, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(y=None), INV), (dict(y=P + 10 * STEP + 1), ALI), (dict(state_out=P + 11 * STEP + 2), ALI),
    (dict(state_in=P + 9 * STEP + 1), ALI), (dict(states=P + 12 * STEP + 4), ALI), (dict(ws=P + 24 * STEP + 8), ALI),
    (dict(y=P + 100), INV), (dict(y=P + 3 * STEP), INV), (dict(state_out=P + 10 * STEP), INV), (dict(states=P + 11 * STEP), INV),
    (dict(state_out=P + 9 * STEP + 16), INV), (dict(y=P + 9 * STEP), INV), (dict(states=P + 9 * STEP), INV),
    (dict(ws=P, L_=5000), INV), (dict(ws=P + 9 * STEP, L_=5000), INV), (dict(lengths=P + 10 * STEP + 8), INV), (dict(ws=None, L_=5000), WS),
    (dict(need=64, L_=5000), WS)])
def test_scan_forward_arguments(kw, status):
    assert scan(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(states=None), INV), (dict(dy=None), INV), (dict(dx=None), INV), (dict(ddelta=None), INV), (dict(dA=None), INV),
    (dict(db=None), INV), (dict(dc=None), INV), (dict(z=None), INV), (dict(dx=P + 15 * STEP + 1), ALI),
    (dict(dA=P + 17 * STEP + 2), ALI), (dict(states=P + 12 * STEP + 8), ALI), (dict(dx=P + 16 * STEP), INV),
    (dict(dz=P + 13 * STEP), INV), (dict(db=P + 19 * STEP + 2), INV), (dict(d_state_in=P + 14 * STEP), INV),
    (dict(dA=P + 2 * STEP), INV), (dict(dx=P + 12 * STEP + 64), INV), (dict(ws=P + 12 * STEP), INV), (dict(ws=None), WS),
    (dict(need=1024), WS)])
def test_scan_backward_arguments(kw, status):
    assert scan(back=True, **kw) == status


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(), dict(state_out=P + 9 * STEP), dict(state_in=None, state_out=None, states=None, D=None, z=None,
                                                                           bias=None, lengths=None), dict(B=0), dict(L_=0),
                                dict(L_=0, x=None, delta=None, b=None, c=None, y=None), dict(N=1), dict(N=64), dict(bs=(0, 0, 0)),
                                dict(xs=(0, 0))])
def test_scan_arguments_that_pass(kw):
    assert scan(**kw) == DEV


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(), dict(dz=None, z=None), dict(dD=None, dbias=None, d_state_in=None, d_state_out=None), dict(B=0),
                                dict(L_=0)])
def test_scan_backward_arguments_that_pass(kw):
    assert scan(back=True, **kw) == DEV


def test_scan_sizes():
    ws = lambda **k: L.eqlinear_selective_scan_workspace_bytes(ctypes.byref(scan_shape(**k)))
    bw = lambda **k: L.eqlinear_selective_scan_backward_workspace_bytes(ctypes.byref(scan_shape(**k)))
    st = lambda **k: L.eqlinear_selective_scan_states_bytes(ctypes.byref(scan_shape(**k)))
    assert ws(L_=1) == 0 and ws(B=0) == 0  # few tokens are one chunk
    assert ws(L_=5000) > 0  # few columns and many tokens are split
    # a state of 4-byte values, N rounded up, each run of 8 tokens
    assert st(C=32, T=2, G=1, N=16, L_=32) == 2 * 4 * 64 * 16 * 4
    assert st(C=32, T=2, G=1, N=16, L_=33) == 2 * 5 * 64 * 16 * 4
    assert bw(L_=5000) > ws(L_=5000) and bw() % 256 == 0
    for bad in (dict(N=65), dict(T=17), dict(dt=4), dict(G=7)):
        assert ws(**bad) == bw(**bad) == st(**bad) == 0


# ---- causal convolution ----

def conv(shape=True, back=False, need=None, B=2, L_=300, C=12, T=4, W=4, act=L.EQL_ACT_SILU, dt=L.EQL_F16, reserved=0, xs=None, **kw):
    at = {n: P + i * STEP for i, n in enumerate(("x", "w", "bias", "lengths", "state_in", "y", "state_out", "dy", "d_state_out", "dx",
                                                 "dw", "db", "d_state_in", "ws"))}
    at.update(kw)
    s = L.ConvShape(B, L_, C, T, W, act, dt, reserved, xs or (C * T * L_, C * T))
    ref = ctypes.byref(s) if shape else None
    g = lambda *n: [at[k] for k in n]
    if back:
        nws = L.eqlinear_causal_conv_backward_workspace_bytes(ref) if need is None else need
        return L.eqlinear_causal_conv_backward(ref, *g("x", "w", "bias", "lengths", "state_in", "dy", "d_state_out", "dx", "dw", "db",
                                                       "d_state_in", "ws"), nws, None)
    return L.eqlinear_causal_conv(ref, *g("x", "w", "bias", "lengths", "state_in", "y", "state_out"), None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), INV), (dict(dt=-1), INV), (dict(B=-1), INV), (dict(W=0), INV), (dict(W=9), UNS), (dict(T=17), UNS),
    (dict(C=65536, T=2), UNS), (dict(act=L.EQL_ACT_GELU), INV), (dict(act=L.EQL_ACT_RELU), INV), (dict(reserved=1), INV),
    (dict(L_=(1 << 30) + 1), UNS), (dict(x=None), INV), (dict(w=None), INV), (dict(x=P + 1), ALI), (dict(w=P + STEP + 1), ALI),
    (dict(lengths=P + 3 * STEP + 2), ALI), (dict(xs=(-8, 48)), INV), (dict(xs=(14400, 1 << 45)), INV)])
@pytest.mark.parametrize("back", [False, True])
def test_conv_arguments(kw, status, back):
    assert conv(back=back, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(y=None), INV), (dict(y=P + 64), INV), (dict(y=P + 4 * STEP), INV), (dict(state_out=P + 4 * STEP + 2), INV),
    (dict(state_out=P + 5 * STEP), INV), (dict(y=P + 5 * STEP + 1), ALI), (dict(state_out=P + STEP), INV)])
def test_conv_forward_arguments(kw, status):
    assert conv(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INV), (dict(dx=None), INV), (dict(dw=None), INV), (dict(dx=P + 7 * STEP), INV), (dict(dw=P + STEP), INV),
    (dict(d_state_in=P + 8 * STEP), INV), (dict(db=P + 10 * STEP + 2), INV), (dict(dx=P + 9 * STEP + 1), ALI), (dict(ws=None), WS),
    (dict(need=16), WS), (dict(ws=P + 13 * STEP + 4), ALI), (dict(ws=P + 9 * STEP), INV)])
def test_conv_backward_arguments(kw, status):
    assert conv(back=True, **kw) == status


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(), dict(state_out=P + 4 * STEP), dict(bias=None, lengths=None, state_in=None, state_out=None), dict(W=1),
                                dict(W=8), dict(B=0), dict(L_=0, x=None, y=None), dict(xs=(0, 0))])
def test_conv_arguments_that_pass(kw):
    assert conv(**kw) == DEV
    assert conv(back=True, **{k: v for k, v in kw.items() if k not in ("y", "state_out")}) == DEV


# ---- residual norm ----

RES_IN = ("x", "u", "w", "b", "scale", "gate", "pw", "pb")


def res(shape=True, back=False, need=None, B=2, L_=50, C=12, T=4, kind=L.EQL_NORM_LAYER, dt=L.EQL_F16, eps=1e-6, reserved=0, **kw):
    names = RES_IN + ("r", "h", "dr", "dh", "dx", "du", "dw", "db", "ds", "dg", "dpw", "dpb", "ws")
    at = {n: P + i * STEP for i, n in enumerate(names)}
    at.update(kw)
    s = L.ResidualShape(B, L_, C, T, kind, dt, eps, reserved)
    ref = ctypes.byref(s) if shape else None
    g = lambda *n: [at[k] for k in n]
    if back:
        nws = L.eqlinear_residual_norm_backward_workspace_bytes(ref) if need is None else need
        return L.eqlinear_residual_norm_backward(ref, *g("x", "u", "w", "scale", "gate", "pw", "pb", "dr", "dh", "dx", "du", "dw", "db",
                                                         "ds", "dg", "dpw", "dpb", "ws"), nws, None)
    return L.eqlinear_residual_norm(ref, *g(*RES_IN, "r", "h"), None)


ALONE = dict(u=None, scale=None, gate=None, pw=None, pb=None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), INV), (dict(dt=3), INV), (dict(B=-1), INV), (dict(C=0), INV), (dict(kind=2), INV), (dict(eps=-1.0), INV),
    (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV), (dict(reserved=1), INV), (dict(T=17), UNS), (dict(C=8193, T=1), UNS),
    (dict(C=1025, T=8), UNS), (dict(B=1 << 20, L_=1 << 20), UNS), (dict(x=None), INV), (dict(u=None), INV),
    (dict(pw=None), INV), (dict(x=P + 1), ALI), (dict(gate=P + 5 * STEP + 1), ALI)])
@pytest.mark.parametrize("back", [False, True])
def test_residual_arguments(kw, status, back):
    assert res(back=back, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(r=None), INV), (dict(h=None), INV), (dict(w=None), INV), (dict(ALONE), INV), (dict(ALONE, r=None, w=None, b=None), INV),
    (dict(r=P), INV), (dict(h=P + STEP), INV), (dict(h=P + 8 * STEP + 64), INV), (dict(r=P + 5 * STEP), INV), (dict(h=P + 9 * STEP + 1), ALI)])
def test_residual_forward_arguments(kw, status):
    assert res(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(w=None), INV), (dict(scale=None), INV), (dict(gate=None), INV), (dict(ALONE), INV), (dict(dx=P + STEP), INV),
    (dict(dx=P + 10 * STEP), INV), (dict(du=P + 12 * STEP + 2), INV), (dict(dw=P + 15 * STEP), INV), (dict(dg=P + 5 * STEP), INV),
    (dict(ws=None), WS), (dict(need=64), WS), (dict(ws=P + 12 * STEP), INV), (dict(ws=P + 20 * STEP + 4), ALI)])
def test_residual_backward_arguments(kw, status):
    assert res(back=True, **kw) == status


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(), dict(ALONE, r=None), dict(b=None, pb=None), dict(w=None, b=None, h=None), dict(B=0), dict(L_=0),
                                dict(C=8192, T=1), dict(C=1, T=1), dict(kind=L.EQL_NORM_RMS, eps=0.0)])
def test_residual_arguments_that_pass(kw):
    assert res(**kw) == DEV


@needs_no_gpu
@pytest.mark.parametrize("kw", [dict(), dict(dr=None), dict(dh=None), dict(dx=None, du=None, dw=None), dict(gate=None, dg=None), dict(B=0),
                                dict(ALONE, du=None, ds=None, dg=None, dpw=None, dpb=None)])
def test_residual_backward_arguments_that_pass(kw):
    assert res(back=True, **kw) == DEV
