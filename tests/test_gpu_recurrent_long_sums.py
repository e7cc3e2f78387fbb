"""Digits of the parameters' gradients of the convolution and of the residual norm over many sequences and many rows.

All terms are 13/9 in fp32: added to itself n times one after the other it is off by 4.6e-5 (n = 4,096), 6.1e-5 (8,192),
1.4e-4 (16,384) and 4.9e-4 (65,536).  An addition rounds by 2^-24 of its sum at most, so a sum is off by 2^-24 times the
number of additions in a row that its longest way takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TERM = 1.4444444179534912
STEP = 2.0 ** -24


def off(got, n):
    return ((got.detach().double() - n * TERM).abs() / (n * TERM)).max().item()


def test_convolution_of_many_sequences():
    """2^20 sequences of a token: a row of sums each, which 64 threads add: 4 columns of a vector, 256 times 64 rows, 4
    sums of a thread, 16 threads and 4 runs of columns."""
    from paper_2607_21271_amd.scan import causal_conv
    B, C, T = 1 << 20, 2, 16
    x = torch.ones(1, 1, C, T, device="cuda").expand(B, 1, C, T)
    w, b = torch.ones(C, 1, device="cuda", requires_grad=True), torch.zeros(C, device="cuda", requires_grad=True)
    dy = torch.full((B, 1, C, T), TERM, device="cuda")
    for g in torch.autograd.grad(causal_conv(x, w, b), (w, b), dy):
        assert off(g, B * T) <= (4 + 64 + 256 + 4 + 64) * STEP
