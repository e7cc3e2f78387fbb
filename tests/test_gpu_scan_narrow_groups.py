"""Scans of 17 to 32 states in groups of a few columns, whose 16-bit vectors are four elements."""
import pytest
import torch

from test_gpu_scan import check, grads, make

pytestmark = pytest.mark.gpu


# whole vectors of four elements, but not of eight; vectors that end with the group; rows shorter than a vector
@pytest.mark.parametrize("C,T,G", [(4, 1, 1), (12, 1, 1), (3, 4, 1), (8, 3, 2), (5, 4, 5), (20, 1, 1), (5, 1, 1), (7, 2, 1), (3, 1, 1), (18, 1, 2)],
                         ids=lambda v: str(v))
@pytest.mark.parametrize("N", [32, 28, 17])
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_narrow_groups(N, C, T, G, dt):
    for B, L in ((2, 37), (300, 5)):
        t = make(N + C, B, L, C, T, N, G, dt)
        check(t)
        check(t, *grads(7, t, L))
    lengths = torch.tensor([20, 3], dtype=torch.int32).cuda()
    t = make(N, 2, 37, C, T, N, G, dt)
    check(t, *grads(8, t, 37), lengths=lengths)
