"""Outputs of the encoder operators that would overlap themselves, values past the C types, heads of no element: refused
before any launch (CPU); turning in place tells autograd (GPU)."""
import ctypes

import pytest
import torch

from paper_2607_21271_amd import _lib as L
from paper_2607_21271_amd import attention, rotary

P, Q, R, S, W = 1 << 20, 1 << 30, 1 << 36, 1 << 40, 1 << 41  # never dereferenced


# y of [2, 5, 3, 8 * 4]: sequences, tokens, heads on top of one another, a token's heads past the next token
@pytest.mark.parametrize("ys", [(0, 96, 32), (480, 0, 32), (480, 96, 0), (480, 64, 32), (96, 96, 32), (32, 32, 320)])
def test_rotary_output_apart(ys):
    sh = L.RotaryShape(2, 5, 3, 8, 4, 2, (2, 1, 0, 0), 0, 0, 0, L.EQL_F16, (480, 96, 32), ys, (10, 2))
    assert L.eqlinear_rotary(ctypes.byref(sh), P, Q, Q + (1 << 20), R, None) == L.EQL_ERR_INVALID_ARG
    same = L.RotaryShape(2, 5, 3, 8, 4, 2, (2, 1, 0, 0), 0, 0, 0, L.EQL_F16, ys, ys, (10, 2))
    assert L.eqlinear_rotary(ctypes.byref(same), P, Q, Q + (1 << 20), P, None) == L.EQL_ERR_INVALID_ARG


@pytest.mark.parametrize("which", range(4))
def test_window_attention_outputs_apart(which):
    q, k = (64 * 256, 256, 64), (64 * 128, 128, 64)
    st = [q, q, k, k]  # o, dq, dk, dv
    st[which] = (0,) + st[which][1:]
    sh = L.WindowShape(2, 64, 64, -1, -1, 0, 4, 2, 64, L.EQL_F16, 0.125, 0, q, k, k, st[0], q, *st[1:])
    if which == 0:
        assert L.eqlinear_window_attention(ctypes.byref(sh), P, Q, Q + (1 << 28), None, None, R, None, None, 0,
                                           None) == L.EQL_ERR_INVALID_ARG
    else:
        assert L.eqlinear_window_attention_backward(
            ctypes.byref(sh), P, Q, Q + (1 << 28), None, None, R, W, S, S + (1 << 28), S + (2 << 28), S + (3 << 28), W, 0,
            None) == L.EQL_ERR_INVALID_ARG


def test_values_past_the_c_types_and_empty_heads():
    f = attention._check_shapes
    q, k = (2, 5, 4, 64), (2, 7, 2, 64)
    f(q, k, k, (1 << 63) - 1, -1, 0)
    for a in ((1 << 63, -1, 0), (-1, 1 << 64, 0), (-1, -1, 1 << 63)):
        with pytest.raises(ValueError):
            f(q, k, k, *a)
    with pytest.raises(ValueError):
        attention.window_attention(torch.zeros(2, 5, 4, 0), torch.zeros(2, 7, 2, 0), torch.zeros(2, 7, 2, 0))
    with pytest.raises(ValueError):
        attention.packed_window_attention(torch.zeros(2, 5, 3, 0), 1)


@pytest.mark.gpu
def test_turning_in_place():
    freqs = rotary.axis_frequencies((4,), device="cuda")
    pos = torch.arange(5, dtype=torch.int32, device="cuda")[:, None]
    with pytest.raises(RuntimeError):
        rotary.rotary_axes_(torch.ones(1, 5, 3, 8, device="cuda").expand(2, 5, 3, 8), pos, freqs, (4,))
    a = torch.ones(2, 5, 3, 8, device="cuda", requires_grad=True)
    x = torch.randn(2, 5, 3, 8, device="cuda")
    y = (a * x).sum()  # keeps x for the gradient of a
    rotary.rotary_axes_(x[:, 1:], pos[1:], freqs, (4,))
    with pytest.raises(RuntimeError):
        y.backward()
    with torch.inference_mode():
        z = torch.ones(2, 5, 3, 8, device="cuda")
        assert rotary.rotary_axes_(z, pos, freqs, (4,)) is z
