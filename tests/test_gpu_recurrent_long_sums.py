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


def test_norm_of_many_rows():
    """2^20 rows of 1,032 columns: a thread adds 4 columns of a channel, 256 rows of its workgroup's strip, and 64 threads the
    4,096 strips: 64 of them, 4 sums of a thread, 16 threads and 2 runs of columns."""
    from paper_2607_21271_amd.norm import residual_norm
    B, C, T = 1 << 20, 129, 8
    x = torch.zeros(1, B, C, T, device="cuda")
    w, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda", requires_grad=True)
    h = residual_norm(x, weight=w, bias=b)[1]
    g, = torch.autograd.grad(h, b, torch.full_like(x, TERM))
    del x, h
    torch.cuda.empty_cache()
    assert off(g, B * T) <= (4 + 256 + 64 + 4 + 32) * STEP


@pytest.mark.parametrize("post", [0, 1])
def test_norm_of_many_sequences(post):
    """2^22 sequences of a token with gates of their own: a thread has 65,536 of them, 64 at a time, after the columns of a
    channel, and 64 threads follow."""
    from paper_2607_21271_amd.norm import residual_norm
    B, C, T = 1 << 22, 2, 8
    one = lambda *s: torch.ones(*s, device="cuda")
    x, u, gate = torch.zeros(B, 1, C, T, device="cuda"), one(B, 1, C, T), one(B, C)
    scale = one(C).requires_grad_()
    pw, pb = (one(C).requires_grad_(), one(C).requires_grad_()) if post else (None, None)
    r = residual_norm(x, u, scale=scale, gate=gate, post_weight=pw, post_bias=pb)[0]
    want = [scale, pb] if post else [scale]  # (the norm of equal elements is 0, so that v is post_bias)
    for g in torch.autograd.grad(r, want, torch.full_like(x, TERM)):
        assert off(g, B * T) <= (8 + 8 + 64 + 1024 + 64) * STEP
    torch.cuda.empty_cache()
