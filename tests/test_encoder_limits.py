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
