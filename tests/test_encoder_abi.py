"""Argument checks of the encoder operators' C entry points, which come before any HIP call (CPU)."""
import ctypes
import os
import re

import pytest

from paper_2607_21271_amd import _lib as L

P, Q, R, S, W = 1 << 20, 1 << 30, 1 << 36, 1 << 40, 1 << 41  # never dereferenced
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "eqlinear_encoder.h")).read()
    names = sorted(set(re.findall(r"\b(eqlinear_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert len(names) == 9
    for n in names:
        assert hasattr(L.lib(), n) and n in L.SIGNATURES and callable(getattr(L, n)), n
    assert L.eqlinear_abi_version() >= 10


def rot(x=P, pos=Q, freqs=Q + (1 << 20), y=R, B=2, L_=5, heads=3, dh=8, T=4, sections=(2, 1), il=0, dt=L.EQL_F16, xs=None,
        ys=None, shape=True):
    s = tuple(sections) + (0,) * (4 - len(sections)) if len(sections) <= 4 else sections[:4]
    st = (heads * dh * T * L_, heads * dh * T, dh * T)
    sh = L.RotaryShape(B, L_, heads, dh, T, len(sections), s, 0, il, 0, dt, xs or st, ys or st, (L_ * 2, 2))
    return L.eqlinear_rotary(ctypes.byref(sh) if shape else None, x, pos, freqs, y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), L.EQL_ERR_INVALID_ARG), (dict(dt=3), L.EQL_ERR_INVALID_ARG), (dict(B=-1), L.EQL_ERR_INVALID_ARG),
    (dict(heads=0), L.EQL_ERR_INVALID_ARG), (dict(sections=(3, 2)), L.EQL_ERR_INVALID_ARG),
    (dict(sections=(0, 0)), L.EQL_ERR_INVALID_ARG), (dict(sections=(5, -4)), L.EQL_ERR_INVALID_ARG),
    (dict(sections=(1,) * 5), L.EQL_ERR_UNSUPPORTED), (dict(T=17), L.EQL_ERR_UNSUPPORTED),
    (dict(dh=1024, T=2), L.EQL_ERR_UNSUPPORTED), (dict(x=None), L.EQL_ERR_INVALID_ARG),
    (dict(freqs=None), L.EQL_ERR_INVALID_ARG), (dict(pos=None), L.EQL_ERR_INVALID_ARG),
    (dict(x=P + 1), L.EQL_ERR_ALIGNMENT), (dict(pos=Q + 2), L.EQL_ERR_ALIGNMENT),
    (dict(y=P + 32), L.EQL_ERR_INVALID_ARG), (dict(y=P, ys=(480, 96, 33)), L.EQL_ERR_INVALID_ARG),
    (dict(y=Q), L.EQL_ERR_INVALID_ARG), (dict(xs=(-480, 96, 32)), L.EQL_ERR_INVALID_ARG)])
def test_rotary_arguments(kw, status):
    assert rot(**kw) == status


def win(q=P, k=Q, v=Q + (1 << 28), o=R, lse=None, ws=None, nws=0, B=2, Lq=64, Lk=64, H=4, Hkv=2, D=64, left=-1, right=-1,
        sinks=0, dt=L.EQL_F16, scale=0.125, qs=None, ks=None, reserved=0, lengths=None, grads=None):
    st = lambda n, l: (n * D * l, n * D, D)
    none = (0, 0, 0)
    q_s, k_s = qs or st(H, Lq), ks or st(Hkv, Lk)
    g = (st(H, Lq), st(H, Lq), st(Hkv, Lk), st(Hkv, Lk)) if grads else (none,) * 4
    sh = L.WindowShape(B, Lq, Lk, left, right, sinks, H, Hkv, D, dt, scale, reserved, q_s, k_s, k_s, st(H, Lq), *g)
    if grads:
        do, dq, dk, dv = grads
        return L.eqlinear_window_attention_backward(ctypes.byref(sh), q, k, v, lengths, None, o, lse, do, dq, dk, dv, ws,
                                                    nws, None)
    return L.eqlinear_window_attention(ctypes.byref(sh), q, k, v, lengths, None, o, lse, ws, nws, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=5), L.EQL_ERR_INVALID_ARG), (dict(B=-1), L.EQL_ERR_INVALID_ARG), (dict(H=3), L.EQL_ERR_INVALID_ARG),
    (dict(left=-2), L.EQL_ERR_INVALID_ARG), (dict(sinks=-1), L.EQL_ERR_INVALID_ARG),
    (dict(scale=0.0), L.EQL_ERR_INVALID_ARG), (dict(scale=float("nan")), L.EQL_ERR_INVALID_ARG),
    (dict(scale=float("inf")), L.EQL_ERR_INVALID_ARG), (dict(reserved=1), L.EQL_ERR_INVALID_ARG),
    (dict(D=136), L.EQL_ERR_UNSUPPORTED), (dict(D=60), L.EQL_ERR_UNSUPPORTED),
    (dict(D=6, dt=L.EQL_F32), L.EQL_ERR_UNSUPPORTED), (dict(Lk=(1 << 28) + 1), L.EQL_ERR_UNSUPPORTED),
    (dict(Lq=1 << 28), L.EQL_ERR_UNSUPPORTED), (dict(q=None), L.EQL_ERR_INVALID_ARG), (dict(v=None), L.EQL_ERR_INVALID_ARG),
    (dict(o=P + 64), L.EQL_ERR_INVALID_ARG), (dict(k=Q + 8), L.EQL_ERR_ALIGNMENT),
    (dict(qs=(16384, 260, 64)), L.EQL_ERR_ALIGNMENT), (dict(lengths=P + 2), L.EQL_ERR_ALIGNMENT),
    (dict(ks=(-8192, 128, 64)), L.EQL_ERR_INVALID_ARG),
    (dict(Lq=1, Lk=100000, B=1), L.EQL_ERR_WORKSPACE),
    (dict(Lq=1, Lk=100000, B=1, ws=W, nws=64), L.EQL_ERR_WORKSPACE)])
def test_window_attention_arguments(kw, status):
    assert win(**kw) == status


G = (S, S + (1 << 28), S + (2 << 28), S + (3 << 28))


@pytest.mark.parametrize("kw,status", [
    (dict(grads=G), L.EQL_ERR_INVALID_ARG),                                   # no lse
    (dict(grads=G, lse=W), L.EQL_ERR_WORKSPACE), (dict(grads=(None,) + G[1:], lse=W), L.EQL_ERR_INVALID_ARG),
    (dict(grads=G[:3] + (Q + 4096,), lse=W), L.EQL_ERR_INVALID_ARG),          # dv inside k
    (dict(grads=G[:1] + (S + 256,) + G[2:], lse=W), L.EQL_ERR_INVALID_ARG),   # dq inside do
    (dict(grads=G[:2] + (G[2] + 4, G[3]), lse=W), L.EQL_ERR_ALIGNMENT)])
def test_window_attention_backward_arguments(kw, status):
    assert win(**kw) == status


def test_window_attention_workspace():
    def need(f, **kw):
        a = dict(B=1, Lq=1, Lk=1 << 16, left=-1, right=-1, sinks=0, H=4, Hkv=2, D=64, dt=L.EQL_F16)
        a.update(kw)
        n = (0, 0, 0)
        return f(ctypes.byref(L.WindowShape(a["B"], a["Lq"], a["Lk"], a["left"], a["right"], a["sinks"], a["H"], a["Hkv"],
                                            a["D"], a["dt"], 1.0, 0, n, n, n, n, n, n, n, n)))
    fwd, bwd = L.eqlinear_window_attention_workspace_bytes, L.eqlinear_window_attention_backward_workspace_bytes
    assert need(fwd) > 0 and need(fwd, B=0) == 0 and need(fwd, D=7) == 0 and need(fwd, Lq=4096, Lk=4096, B=64) == 0
    assert need(bwd, Lq=4096, Lk=4096) >= 4096 * 4 * 4 and need(bwd, B=0) == 0
    assert need(bwd, Lq=1 << 16, left=100, right=0, sinks=4) > need(bwd, Lq=1 << 16, left=100, right=0)  # parts of sink tiles


def gn(x=P, w=Q, b=Q + 4096, y=R, stats=None, ws=W, nws=1 << 30, B=2, S_=9, T=4, C=24, G=4, eps=1e-5, act=1, dt=L.EQL_F16):
    return L.eqlinear_group_norm_act(x, w, b, y, stats, ws, nws, B, S_, T, C, G, eps, act, dt, None)


def gnb(x=P, w=Q, b=Q + 4096, stats=Q + 8192, dy=R, dx=S, dw=Q + 16384, db=Q + 20480, ws=W, nws=1 << 30, B=2, S_=9, T=4,
        C=24, G=4, act=1, dt=L.EQL_F16):
    return L.eqlinear_group_norm_act_backward(x, w, b, stats, dy, dx, dw, db, ws, nws, B, S_, T, C, G, act, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=9), L.EQL_ERR_INVALID_ARG), (dict(G=5), L.EQL_ERR_INVALID_ARG), (dict(G=0), L.EQL_ERR_INVALID_ARG),
    (dict(B=-1), L.EQL_ERR_INVALID_ARG), (dict(act=4), L.EQL_ERR_INVALID_ARG), (dict(x=None), L.EQL_ERR_INVALID_ARG),
    (dict(w=None), L.EQL_ERR_INVALID_ARG), (dict(T=17), L.EQL_ERR_UNSUPPORTED), (dict(C=2050, G=1025), L.EQL_ERR_UNSUPPORTED),
    (dict(x=P + 8), L.EQL_ERR_ALIGNMENT), (dict(b=Q + 4097), L.EQL_ERR_ALIGNMENT),
    (dict(ws=None, S_=1 << 16), L.EQL_ERR_WORKSPACE), (dict(nws=8, S_=1 << 16), L.EQL_ERR_WORKSPACE)])
def test_group_norm_arguments(kw, status):
    assert gn(**kw) == status
    assert gnb(**kw) == status


def test_group_norm_own_arguments():
    assert gn(eps=-1.0) == L.EQL_ERR_INVALID_ARG and gn(eps=float("nan")) == L.EQL_ERR_INVALID_ARG
    assert gn(y=P + 16) == L.EQL_ERR_INVALID_ARG
    assert gnb(dx=P + 16) == L.EQL_ERR_INVALID_ARG and gnb(dw=Q) == L.EQL_ERR_INVALID_ARG
    assert gnb(db=Q + 16384) == L.EQL_ERR_INVALID_ARG and gnb(stats=None) == L.EQL_ERR_INVALID_ARG
    ws = L.eqlinear_group_norm_act_workspace_bytes
    assert ws(2, 1 << 16, 4, 24, 4, L.EQL_F16) > 0 and ws(0, 1 << 16, 4, 24, 4, L.EQL_F16) == 0 and ws(2, 9, 4, 24, 5, L.EQL_F16) == 0
