"""Refusals of the encoder operators' torch wrappers, which come before any launch, and their host-side helpers (CPU)."""
import pytest
import torch

from paper_2607_21271_amd import attention, norm, rotary


def z(*s, dt=torch.float16):
    return torch.zeros(*s, dtype=dt)


def test_window_attention_refusals():
    f = attention.window_attention
    q, k = z(2, 5, 4, 64), z(2, 7, 2, 64)
    for args, kw, err in [
            ((z(2, 5, 4, 64, dt=torch.float64), k, k), {}, TypeError), ((q, k, z(2, 7, 2, 64, dt=torch.float32)), {}, TypeError),
            ((q[0], k, k), {}, ValueError), ((q, k, z(2, 7, 1, 64)), {}, ValueError), ((q, z(1, 7, 2, 64), z(1, 7, 2, 64)), {}, ValueError),
            ((q, z(2, 7, 3, 64), z(2, 7, 3, 64)), {}, ValueError), ((q, z(2, 7, 2, 32), z(2, 7, 2, 32)), {}, ValueError),
            ((q, k, k), dict(left=-2), ValueError), ((q, k, k), dict(sinks=-1), ValueError), ((q, k, k), {}, ValueError)]:
        with pytest.raises(err):
            f(*args, **kw)  # the last: tensors of the CPU
    with pytest.raises(ValueError):
        attention._check_spans(2, q, torch.zeros(2, dtype=torch.int64), None)
    with pytest.raises(ValueError):
        attention._check_spans(2, q, None, torch.zeros(3, dtype=torch.int32))


def test_packed_attention_refusals():
    f = attention.packed_window_attention
    for x, hkv in ((z(2, 5, 4, 64), 2), (z(2, 5, 7, 64), 2), (z(2, 5, 4), 1), (z(2, 5, 4, 64), 0), (z(2, 5, 4, 64), 1)):
        with pytest.raises(ValueError):
            f(x, hkv)


def test_rotary_refusals():
    f = rotary.rotary_axes
    x, p, w = z(2, 5, 3, 32), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(3)
    for args, kw, err in [
            ((x.double(), p, w, (2, 1)), dict(T=4), TypeError), ((x[0], p, w, (2, 1)), dict(T=4), ValueError),
            ((x, p, w, (2, 1)), dict(T=3), ValueError), ((x, p, w, (3, 2)), dict(T=4), ValueError),
            ((x, p, w, (2, -1)), dict(T=4), ValueError), ((x, p[:4], w, (2, 1)), dict(T=4), ValueError),
            ((x, p.long(), w, (2, 1)), dict(T=4), TypeError), ((x, p, w[:2], (2, 1)), dict(T=4), ValueError),
            ((x, p, w.double(), (2, 1)), dict(T=4), ValueError), ((x, p, w, (2, 1)), dict(T=4), ValueError)]:
        with pytest.raises(err):
            f(*args, **kw)
    with pytest.raises(ValueError):
        rotary.axis_frequencies((2, 1), theta=(1e4,))


def test_rotary_helpers():
    f = rotary.axis_frequencies((2, 1), theta=(100.0, 7.0))
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 1.0]))
    p = rotary.grid_positions((2, 3), prefix=1)
    assert p.dtype == torch.int32 and p.tolist() == [[0, 0], [0, 0], [0, 1], [0, 2], [1, 0], [1, 1], [1, 2]]


def test_group_norm_refusals():
    f = norm.group_norm_act
    x, w = z(2, 9, 8, 4), z(8)
    for args, kw, err in [
            ((x.double(), w, w, 2), {}, TypeError), ((x, w.float(), w, 2), {}, TypeError), ((z(8, 4), w, w, 2), {}, ValueError),
            ((x, z(7), w, 2), {}, ValueError), ((x, w, w, 3), {}, ValueError), ((x, w, w, 0), {}, ValueError),
            ((x, w, w, 2), dict(activation="tanh"), ValueError), ((x, w, w, 2), {}, ValueError)]:
        with pytest.raises(err):
            f(*args, **kw)
