"""The scan's gradients of parameters over long chunks of tokens: sums that a wave takes to memory on the way (32 tiles), and the
digits of sums over many tokens and sequences."""
import ctypes

import pytest
import torch

import recurrent_ref as R
from paper_2607_21271_amd import _lib as L

pytestmark = pytest.mark.gpu


def plan(B, Lt, C, T, N, dt=L.EQL_F32):
    """(chunks, tiles of a chunk) of the gradients, from the bytes of their workspace."""
    s = L.ScanShape(B, Lt, C, T, N, 1, 1, dt, (0, 0), (0, 0), (0, 0), (0, 0, 0), (0, 0, 0))
    back = L.eqlinear_selective_scan_backward_workspace_bytes(ctypes.byref(s))
    NL = 1 if N <= 4 else 2 if N <= 8 else 4 if N <= 16 else 8 if N <= 32 else 16
    width, NP, tile, up = 256 // NL, 4 * NL, {1: 4, 2: 8}.get(NL, 16), lambda v: -(-v // 256) * 256
    cols, tiles, found = -(-C * T // width) * width, -(-Lt // tile), set()
    for per in range(1, tiles + 1):
        K = -(-tiles // per)
        fixed = (up(B * K * cols * NP * 4) + up(B * K * cols * 4) if K > 1 else 0) + up(B * K * (N + 2) * cols * 4)
        for P in range(1, 2 * cols * NL // 256 + 1):
            if -(-tiles // K) == per and fixed + (up(B * Lt * P * 2 * NP * 4) if P > 1 else 0) == back:
                found.add((K, per))
    assert len(found) == 1, found
    return found.pop()


class Here:
    """lengths for a reference on the GPU."""

    def __init__(self, t):
        self.cpu = lambda: t


@pytest.mark.parametrize("size,slices", [((2048, 300, 32, 4, 4), 8), ((256, 1100, 32, 8, 16), 16)], ids=["4 states", "16 states"])
@pytest.mark.parametrize("ragged", [0, 1])
def test_sums_are_taken_to_memory(size, slices, ragged, monkeypatch):
    """More than 64 tiles a wave: two times a wave adds its sums to memory, and once more at its end.  All terms of dA have one
    sign, and so have those of dD and of the bias's gradient, so that none can be lost or counted twice."""
    from paper_2607_21271_amd.scan import selective_scan
    B, Lt, C, T, N = size
    K, per = plan(*size)
    assert K == 1 and per > 64
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.rand(*s, generator=g, device="cuda") + 0.25
    t = dict(x=n(B, Lt, C, T), delta=n(B, Lt, C, T), A=-n(C, N), Bt=n(B, Lt, 1, N), Ct=n(B, Lt, 1, N), D=n(C), z=n(B, Lt, C, T),
             delta_bias=n(C) - 3)
    dy = n(B, Lt, C, T)
    lengths = torch.randint(Lt // 4, Lt + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if ragged else None
    wide = {k: t[k].requires_grad_() for k in ("A", "D", "delta_bias")}
    got = torch.autograd.grad(selective_scan(**t, lengths=lengths), list(wide.values()), dy)
    t = {k: v.detach() for k, v in t.items()}
    monkeypatch.setattr(R, "_d", lambda v: None if v is None else v.detach().double())
    want = [[0.0, 0.0] for _ in got]
    with torch.device("cuda"):
        for i in range(slices):
            s = slice(i * B // slices, (i + 1) * B // slices)
            part = R.scan(**{k: v[s] if v.dim() == 4 else v for k, v in t.items()}, dy=dy[s],
                          lengths=None if lengths is None else Here(lengths[s].long()))
            for w, k in zip(want, ("dA", "dD", "dbias")):
                w[0], w[1] = w[0] + part[k][0], w[1] + part[k][1]
            del part
    for v, w, k in zip(got, want, ("dA", "dD", "dbias")):
        R.within(k, v, w[0].cpu(), (w[1] + 64 * 2.0 ** -24 * w[0].abs()).cpu())
    torch.cuda.empty_cache()


# 13/9: added to itself n times one after the other it is off by 1.8e-5 (n = 2,048) and 4.6e-5 (4,096)
TERM = 1.4444444179534912


@pytest.mark.parametrize("B,Lt,C,T", [(256, 16384, 32, 8), (1 << 16, 2, 4, 16)], ids=["tokens", "sequences"])
def test_digits_of_long_sums(B, Lt, C, T):
    """dD and ddelta_bias of equal terms, over 16,384 tokens a wave and over 65,536 sequences.  An addition rounds by 2^-24 of
    its sum at most.  Over tokens a lane adds 64 terms (32 tiles of two) before three steps over lanes, 32 such sums meet in
    memory, and 8 sequences a thread and 256 threads follow: 64 + 3 + 32 + 8 + 8 additions in a row.  Over sequences a thread has 4,096
    sums of two tokens, taken 64 at a time: 2 + 3 + 64 + 64 + 8.  No more than 160 either way."""
    from paper_2607_21271_amd.scan import selective_scan
    N = 16
    if Lt > 1000:
        K, per = plan(B, Lt, C, T, N)
        assert K == 1 and per == 1024
    one = lambda v, *s: torch.full((1,) * len(s), v, device="cuda").expand(*s)
    # decays of exp(-1e4 d) = 0: every token's gradient is its own.  ddelta = x sum_n b c dy
    row = lambda v, *s: torch.full((1, 1, *s), v, device="cuda").expand(B, Lt, *s)
    x, delta = row(TERM, C, T), row(1.0, C, T)
    Bt, Ct = row(0.25, 1, N), row(0.25, 1, N)  # (sum_n b c = 1)
    A, D, bias = torch.full((C, N), -1e4, device="cuda"), torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")
    dy = torch.ones(B, Lt, C, T, device="cuda")
    D.requires_grad_()
    bias.requires_grad_()
    dD, db = torch.autograd.grad(selective_scan(x, delta, A, Bt, Ct, D, delta_bias=bias, softplus=False), (D, bias), dy)
    want = B * Lt * T * TERM
    bound = 160 * 2.0 ** -24 * want
    assert (dD.double() - want).abs().max() <= bound, ((dD.double() - want).abs().max().item() / want)
    assert (db.double() - want).abs().max() <= bound, ((db.double() - want).abs().max().item() / want)
    torch.cuda.empty_cache()
