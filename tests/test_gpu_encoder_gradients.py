"""Gradients of windowed attention where sizes or values are extreme, against 64 bits (tests/encoder_ref.py)."""
import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu


def gradients(q, k, v, do, **kw):
    from paper_2607_21271_amd.attention import window_attention
    q, k, v = (t.detach().requires_grad_() for t in (q, k, v))
    o = window_attention(q, k, v, **kw)
    return dict(zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, (q, k, v), do))))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_gradient_without_keys(dt):
    g = torch.Generator().manual_seed(1)
    q, do = (torch.randn(2, 3, 4, 64, generator=g).to(R.DT[dt]).cuda() for _ in range(2))
    k = torch.zeros(2, 0, 2, 64, dtype=R.DT[dt], device="cuda")
    got = gradients(q, k, k.clone(), do, sinks=2)
    assert (got["o"] == 0).all() and (got["dq"] == 0).all() and got["dk"].shape == got["dv"].shape == k.shape


def f16(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).half().cuda()


def compare(q, k, v, do, **kw):
    got, want = gradients(q, k, v, do, **kw), R.attention(q, k, v, do, **kw)
    for n, t in got.items():
        assert torch.isfinite(t).all(), n
        R.within(n, t, *want[n])


@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("L,kw", [(2, {}), (150, dict(right=0)), (333, dict(left=40, right=7, sinks=2))])
def test_fp16_large_values(L, kw, D):
    """Values of 4,000 and small gradients: score gradients of hundreds of thousands times the largest |do|."""
    v = torch.sign(f16(13, 1, L, 1, D)) * 4000.0
    if L == 2:
        v[0, 0], v[0, 1] = 4000.0, -4000.0
        do = torch.full((1, L, 2, D), 1e-3, dtype=torch.float16, device="cuda")
    else:
        do = f16(14, 1, L, 2, D, scale=1e-3)
    compare(f16(11, 1, L, 2, D, scale=0.5), f16(12, 1, L, 1, D, scale=0.5), v, do, **kw)


@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("row", [0, 70, 199])
def test_fp16_one_large_gradient_beside_small_ones(row, D):
    """A row of 30,000 among rows of 0.01: keys that it does not see keep the bits of their gradients, and so do rows."""
    do = f16(24, 1, 200, 2, D, scale=0.01)
    do[0, row, 1] = 30000.0 * torch.sign(do[0, row, 1])
    compare(f16(21, 1, 200, 2, D), f16(22, 1, 200, 1, D), f16(23, 1, 200, 1, D), do, left=20, right=0)


def test_fp16_gradients_grow_along_the_rows():
    """Rows whose gradients grow by 2^20 from first to last, and shrink: the power of two of a key moves with them."""
    L = 256
    size = torch.logspace(-10, 10, L, base=2.0).cuda()[None, :, None, None]
    for s in (size, size.flip(1)):
        do = (f16(34, 1, L, 1, 64).float() * s).half()
        compare(f16(31, 1, L, 1, 64), f16(32, 1, L, 1, 64), f16(33, 1, L, 1, 64), do, left=50, right=50)


@pytest.mark.parametrize("L,H,D,kw", [(700, 2, 64, {}), (2000, 1, 128, {}), (1500, 1, 96, dict(left=900, right=900)), (509, 3, 40, dict(left=100, right=20))])
def test_full_precision_gradients(L, H, D, kw):
    """2-norm errors of full-precision gradients.  A probability is exp2(c s - lse): below 2^m the logarithm and the
    difference are each rounded by 2^(m - 25) at most, so it is off by 2 ln 2 2^(m - 25) of itself; the sums of products
    add 2^-21 (random signs: sqrt(2000) roundings of 2^-24 of terms, and of D / 2 in the scores)."""
    g = torch.Generator().manual_seed(41)
    q, k, v, do = (torch.randn(1, L, H, D, generator=g).cuda() for _ in range(4))
    got, want = gradients(q, k, v, do, **kw), R.attention(q, k, v, do, **kw)
    bits = 3 if min(L, sum(kw.values()) or L) < 200 else 4  # lse of that many keys and scores of spread one
    bound = 2 * 0.6932 * 2.0 ** (bits - 25) + 2.0 ** -21
    for n in ("o", "dq", "dk", "dv"):
        err = ((got[n].double().cpu() - want[n][0]).norm() / want[n][0].norm()).item()
        assert err <= bound, (n, err, bound)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("L,D,kw", [(400, 64, dict(left=1, right=0)), (400, 64, dict(left=2, right=0)), (300, 128, dict(left=1, right=1)),
                                    (500, 32, dict(left=4, right=0, sinks=1)), (400, 64, dict(left=8, right=8)), (3, 64, {}),
                                    (700, 96, dict(left=-1, right=0)), (400, 64, dict(left=40, right=0))])
def test_gradients_of_rows_that_see_few_keys(L, D, kw, dt):
    """2-norm errors against results rounded once.  A score gradient is rounded once and its sums once, independent
    roundings: sqrt(2); a row's probabilities share an error of at most half that size: sqrt(2.25) = 1.5, and 0.15 for
    the sample (sequences of three tokens: two dozen of them)."""
    g = torch.Generator().manual_seed(51)
    B = 24 if L < 10 else 2
    q, k, v, do = (torch.randn(B, L, 2, D, generator=g).to(R.DT[dt]).cuda() for _ in range(4))
    got, want = gradients(q, k, v, do, **kw), R.attention(q, k, v, do, **kw)
    for n in ("dq", "dk", "dv"):
        w = want[n][0]
        once = (w.to(R.DT[dt]).double() - w).norm()
        err = (got[n].double().cpu() - w).norm()
        assert err <= 1.65 * once, (n, (err / once).item())
