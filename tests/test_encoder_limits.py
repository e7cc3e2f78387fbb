"""Sizes at the ends of what the encoder operators take: no keys, many first tokens, large batches, outputs in one
buffer (CPU: workspace queries and argument checks, which come before any HIP call)."""
import ctypes

import pytest

from paper_2607_21271_amd import _lib as L

NONE = (0, 0, 0)


def window(B, Lq, Lk, H, Hkv, D, left=-1, right=-1, sinks=0, dt=L.EQL_F16):
    return ctypes.byref(L.WindowShape(B, Lq, Lk, left, right, sinks, H, Hkv, D, dt, 0.125, 0, *(NONE,) * 8))


@pytest.mark.parametrize("dt", [L.EQL_F32, L.EQL_F16, L.EQL_BF16])
def test_workspace_without_keys_or_queries(dt):
    need = L.eqlinear_window_attention_backward_workspace_bytes
    rows = 2 * 3 * 4 * 4  # one fp32 a row; no parts
    assert rows <= need(window(2, 3, 0, 4, 2, 64, dt=dt)) <= 4096
    assert need(window(2, 0, 0, 4, 2, 64, dt=dt)) == need(window(2, 0, 5, 4, 2, 64, dt=dt)) == 0
    assert L.eqlinear_window_attention_workspace_bytes(window(2, 3, 0, 4, 2, 64, dt=dt)) == 0


@pytest.mark.parametrize("B,L_,H,D,left,sinks", [
    (4, 8192, 8, 128, 63, 4096), (8, 65536, 8, 128, 63, 1024), (8, 65536, 8, 128, 63, 16384), (1, 1 << 20, 8, 64, 100, 1 << 19),
    (64, 2048, 12, 64, 31, 4), (1, 600, 1, 80, 15, 3), (3, 5000, 5, 96, 0, 700)])
def test_parts_of_the_key_gradient_are_bounded(B, L_, H, D, left, sinks):
    """Parts exist to fill 256 CUs: eight a CU of first tokens and one of other keys, each two fp32 tiles of 128 keys, are
    enough for any shape.  (Beside them two fp32 values a row at most.)"""
    got = L.eqlinear_window_attention_backward_workspace_bytes(window(B, L_, L_, H, H, D, left, 0, sinks))
    assert 0 < got <= 9 * 256 * 2 * 128 * D * 4 + 8 * B * H * (L_ + 128) + 1024


def test_first_tokens_of_few_sequences_are_split():
    need = L.eqlinear_window_attention_backward_workspace_bytes
    assert need(window(1, 8192, 8192, 2, 2, 64, 100, 0, 4)) > need(window(1, 8192, 8192, 2, 2, 64, 100, 0, 0))


# ---- buffers that lie on one another (addresses are never dereferenced) ----------------------------------------------

P, S, W = 1 << 20, 1 << 36, 1 << 41
STEP = 1 << 28


def dense(n, heads, D, T=0):
    return (T or n) * heads * D, heads * D, D


def forward(B=2, L_=64, H=4, Hkv=2, D=64, o=S, lse=None, ws=None, lengths=None, starts=None, Lq=None):
    Lq = Lq or L_
    sh = L.WindowShape(B, Lq, L_, -1, -1, 0, H, Hkv, D, L.EQL_F16, 0.125, 0, dense(Lq, H, D), dense(L_, Hkv, D),
                       dense(L_, Hkv, D), dense(Lq, H, D), *(NONE,) * 4)
    need = L.eqlinear_window_attention_workspace_bytes(ctypes.byref(sh))
    return L.eqlinear_window_attention(ctypes.byref(sh), P, P + STEP, P + 2 * STEP, lengths, starts, o, lse, ws, need, None)


def backward(B=2, L_=64, H=4, Hkv=2, D=64, dq=S, dk=S + STEP, dv=S + 2 * STEP, st=None, lse=W, ws=W + STEP, o=P + 3 * STEP,
             lengths=None, starts=None):
    st = st or (dense(L_, H, D), dense(L_, Hkv, D), dense(L_, Hkv, D))
    sh = L.WindowShape(B, L_, L_, -1, -1, 0, H, Hkv, D, L.EQL_F16, 0.125, 0, dense(L_, H, D), dense(L_, Hkv, D),
                       dense(L_, Hkv, D), dense(L_, H, D), dense(L_, H, D), *st)
    need = L.eqlinear_window_attention_backward_workspace_bytes(ctypes.byref(sh))
    return L.eqlinear_window_attention_backward(ctypes.byref(sh), P, P + STEP, P + 2 * STEP, lengths, starts, o, lse,
                                                P + 4 * STEP, dq, dk, dv, ws, need, None)


PASSED = (L.EQL_ERR_NO_DEVICE,)  # the next thing that is looked at; where there is a GPU these are not called
needs_no_gpu = pytest.mark.skipif(__import__("torch").cuda.device_count() > 0, reason="addresses that hold nothing")
E2 = 2  # bytes of an element


@pytest.mark.parametrize("kw", [
    dict(dk=S + STEP, dv=S + STEP), dict(dq=S, dk=S), dict(dq=S, dv=S + 128), dict(dk=S + STEP, dv=S + STEP + 16),
    dict(ws=P + STEP), dict(ws=S), dict(ws=W), dict(lse=S + 64), dict(lengths=S + 8), dict(starts=S + STEP + 4),
    dict(lengths=W + STEP), dict(o=W + STEP),
    # dq and dk of one packed buffer, one head too close; with a last head on the next token's first
    dict(st=((64 * 8 * 64, 8 * 64, 64),) * 3, dq=S, dk=S + 3 * 64 * E2, dv=S + 6 * 64 * E2),
    dict(st=((64 * 8 * 64, 8 * 64, 64),) * 3, dq=S, dk=S + 4 * 64 * E2, dv=S + 7 * 64 * E2),
    # overlapping spans of other strides
    dict(st=(dense(64, 4, 64), (64 * 512, 512, 64), dense(64, 2, 64)), dk=S + 64)])
def test_gradient_outputs_apart(kw):
    assert backward(**kw) == L.EQL_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(o=S, lse=S), dict(lse=P), dict(lse=P + 2 * STEP + 16), dict(lengths=S), dict(starts=S + 4),
                                dict(lse=W, lengths=W + 4), dict(B=1, L_=100000, Lq=1, ws=S), dict(B=1, L_=100000, Lq=1, ws=P + STEP),
                                dict(B=1, L_=100000, Lq=1, ws=W, lse=W + 32)])
def test_outputs_apart(kw):
    assert forward(**kw) == L.EQL_ERR_INVALID_ARG


@needs_no_gpu
@pytest.mark.parametrize("kw", [
    {}, dict(lengths=W - 4096, starts=W - 2048),
    # one packed buffer: tokens of queries, keys, values; sequences padded; heads before tokens; tokens before sequences
    dict(st=((64 * 8 * 64, 8 * 64, 64),) * 3, dq=S, dk=S + 4 * 64 * E2, dv=S + 6 * 64 * E2),
    dict(st=((64 * 8 * 64 + 24, 8 * 64, 64),) * 3, dq=S, dk=S + 4 * 64 * E2, dv=S + 6 * 64 * E2),
    dict(st=((64 * 8 * 64, 64, 64 * 64),) * 3, dq=S, dk=S + 4 * 64 * 64 * E2, dv=S + 6 * 64 * 64 * E2),
    dict(st=((8 * 64, 2 * 8 * 64, 64),) * 3, dq=S, dk=S + 4 * 64 * E2, dv=S + 6 * 64 * E2),
    dict(st=((8 * 64, 0, 64),) * 3, L_=1, dq=S, dk=S + 4 * 64 * E2, dv=S + 6 * 64 * E2),
    dict(st=((64 * 4 * 64, 4 * 64, 64), (64 * 4 * 64, 4 * 64, 0), (64 * 4 * 64, 4 * 64, 0)), H=2, Hkv=1, dq=S,
         dk=S + 2 * 64 * E2, dv=S + 3 * 64 * E2)])
def test_gradients_may_interleave(kw):
    assert backward(**kw) in PASSED


@needs_no_gpu
def test_outputs_that_are_apart():
    assert forward() in PASSED and forward(lse=W, lengths=W + STEP, starts=W + 2 * STEP) in PASSED
    assert forward(B=1, L_=100000, Lq=1, ws=W, lse=W + STEP) in PASSED


def norm(f, **kw):
    a = dict(x=P, w=P + STEP, b=P + STEP + 4096, y=S, stats=W, ws=W + STEP, B=2, S_=1 << 16, T=4, C=24, G=4)
    a.update(kw)
    shape = (a["B"], a["S_"], a["T"], a["C"], a["G"])
    if f == "forward":
        return L.eqlinear_group_norm_act(a["x"], a["w"], a["b"], a["y"], a["stats"], a["ws"], 1 << 26, *shape, 1e-5, 1,
                                         L.EQL_F16, None)
    g = dict(dy=P + 2 * STEP, dx=S + STEP, dw=S + 2 * STEP, db=S + 2 * STEP + 4096)
    g.update({n: v for n, v in kw.items() if n in g})
    return L.eqlinear_group_norm_act_backward(a["x"], a["w"], a["b"], a["stats"], g["dy"], g["dx"], g["dw"], g["db"], a["ws"],
                                              1 << 26, *shape, 1, L.EQL_F16, None)


@pytest.mark.parametrize("f,kw", [
    ("forward", dict(stats=S)), ("forward", dict(stats=P + STEP)), ("forward", dict(ws=S + 4096)), ("forward", dict(ws=P)),
    ("forward", dict(ws=W)), ("backward", dict(stats=S + STEP + 8)), ("backward", dict(ws=S + 2 * STEP)),
    ("backward", dict(ws=W)), ("backward", dict(ws=P + 2 * STEP)), ("backward", dict(stats=S + 2 * STEP))])
def test_group_norm_buffers_apart(f, kw):
    assert norm(f, **kw) == L.EQL_ERR_INVALID_ARG


@needs_no_gpu
def test_group_norm_buffers_that_are_apart():
    assert norm("forward") in PASSED and norm("backward") in PASSED


# B, S, C, T, groups: groups of one channel in passes; held groups, 2^24 of them; many channels of many sequences
LARGE = [(262144, 16, 32, 1, 32), ((1 << 18) + 5, 1, 512, 1, 64), (16384, 1, 65536, 1, 1024), (1 << 20, 1, 3843, 1, 3),
         (1 << 20, 3, 1024, 2, 1024)]


@needs_no_gpu
@pytest.mark.parametrize("B,S_,C,T,G", LARGE)
def test_group_norm_of_large_batches(B, S_, C, T, G):
    """What the forward takes, the gradient takes; more workgroups than one launch holds are no limit."""
    n = L.eqlinear_group_norm_act_workspace_bytes(B, S_, T, C, G, L.EQL_F16)
    m = L.eqlinear_group_norm_act_backward_workspace_bytes(B, S_, T, C, G, L.EQL_F16)
    T_ = [i << 40 for i in range(1, 11)]
    assert L.eqlinear_group_norm_act(T_[0], T_[1], T_[2], T_[3], T_[4], T_[5], n, B, S_, T, C, G, 1e-5, 0, L.EQL_F16,
                                     None) in PASSED
    assert L.eqlinear_group_norm_act_backward(T_[0], T_[1], T_[2], T_[3], T_[4], T_[5], T_[6], T_[7], T_[8], m, B, S_, T, C,
                                              G, 0, L.EQL_F16, None) in PASSED
