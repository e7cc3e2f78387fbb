"""The scan's carry over chunks of tokens where a chunk's decay as a whole leaves the range of fp32: growing states that are 0 or
tiny, infinite states that decay.  Token by token all of it is finite, or infinite and stays so."""
import pytest
import torch

import recurrent_ref as R
from encoder_ref import DT

pytestmark = pytest.mark.gpu
# a few columns of many tokens, which are cut into chunks; every number of lanes that share columns
SIZES = [(2, 3000, 5, 1, 3, 1), (1, 2500, 8, 2, 8, 2), (1, 4000, 12, 4, 16, 1), (1, 3000, 3, 3, 20, 1), (1, 2000, 4, 1, 64, 1)]


def make(seed, B, L, C, T, N, G, dt="f32"):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: (torch.rand(*s, generator=g) + 0.5).to(DT[dt]).cuda()
    return dict(x=n(B, L, C, T), delta=n(B, L, C, T), A=n(C, N).float(), Bt=n(B, L, G, N), Ct=n(B, L, G, N), D=n(C).float())


def is_cut(t):
    """Whether the plan cuts the call into chunks: only then has the forward a workspace."""
    from paper_2607_21271_amd import scan
    return scan._scan_check(t["x"], t["delta"], t["A"], t["Bt"], t["Ct"], t.get("D"), None, None, False, None).need > 0


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_growth_from_nothing(size, dt):
    """A above 0 and elements of 0 up to the last 20 tokens: the states are 0 until then, however much they would have grown."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(1, *size, dt)
    t["A"] *= 8
    L, n = size[1], 20
    t["x"][:, :-n] = 0
    t["delta"][:, -n:] *= 0.01
    assert is_cut(t)
    with torch.no_grad():
        y, h = selective_scan(**t, softplus=False, return_state=True)
    last = {k: v[:, -n:] if v.dim() == 4 else v for k, v in t.items()}
    want = R.scan(**last, softplus=False)
    assert (y[:, :-n] == 0).all()
    R.within("y", y[:, -n:], *want["y"])
    R.within("state", h, *want["state"])


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gradients_grow_from_nothing(size):
    """The same from the other end: a gradient at the first 20 tokens alone."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(2, *size)
    t["A"] *= 8
    n = 20
    t["x"].zero_()
    t["delta"][:, :n] *= 0.01
    dy = torch.rand(t["x"].shape, generator=torch.Generator().manual_seed(3)).cuda()
    dy[:, n:] = 0
    given = {k: v.detach().requires_grad_() for k, v in t.items()}
    got = dict(zip(given, torch.autograd.grad(selective_scan(**given, softplus=False), list(given.values()), dy)))
    first = {k: v[:, :n] if v.dim() == 4 else v for k, v in t.items()}
    want = R.scan(**first, softplus=False, dy=dy[:, :n])
    for k, name in (("x", "dx"), ("delta", "ddelta"), ("Bt", "dBt"), ("Ct", "dCt")):
        assert (got[k][:, n:] == 0).all(), name
        R.within(name, got[k][:, :n], *want[name])
    for k, name in (("A", "dA"), ("D", "dD")):
        R.within(name, got[k], *want[name])


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_growth_of_tiny_states(size):
    """A state of 2^-120 that grows by 2^160, over the first tile of a cut call, and keeps its digits; and the way back."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(4, *size)
    B, L, C, T, N, G = size
    tile = 4 if N <= 4 else 8 if N <= 8 else 16
    t["x"].zero_()
    t["delta"].zero_()
    t["delta"][:, :tile] = 160 / tile
    t["A"].fill_(0.6931471805599453)
    h0 = (torch.rand(B, C, T, N, generator=torch.Generator().manual_seed(5)) + 0.5).cuda() * 2.0 ** -120
    assert is_cut(t)
    with torch.no_grad():
        h = selective_scan(**t, softplus=False, state=h0, return_state=True)[1]
    grown = torch.exp(t["delta"].double()[0, :tile, 0, 0].sum() * t["A"].double()[0, 0])
    # the growth's exponent 160 holds three roundings, of log2(e), of A times it and of that times the sum of the steps, which is
    # exact: 3 * 160 ln 2 2^-24 of the value; and a few units for the exponential and the products
    off = (480 * 0.694 + 8) * 2.0 ** -24
    assert ((h.double() - h0.double() * grown).abs() <= off * h0.double() * grown).all()
    state = h0.clone().requires_grad_()
    g, = torch.autograd.grad(selective_scan(**t, softplus=False, state=state, return_state=True)[1], state, h0)
    assert ((g.double() - h0.double() * grown).abs() <= off * h0.double() * grown).all()


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_infinite_states_stay_infinite(size):
    """Steps of exp(-20) each: a chunk's decay as a whole is 0 in fp32, and 0 times infinity would be NaN."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(6, *size)
    B, L, C, T, N, G = size
    t["A"].fill_(-20.0)
    t["delta"].fill_(1.0)
    h0 = torch.ones(B, C, T, N, device="cuda")
    h0[:, 0, 0, 0] = float("inf")
    assert is_cut(t)
    with torch.no_grad():
        y, h = selective_scan(**t, softplus=False, state=h0, return_state=True)
    assert (y[:, :, 0, 0] == float("inf")).all() and (h[:, 0, 0, 0] == float("inf")).all()
    assert torch.isfinite(y[:, :, 1:]).all() and torch.isfinite(h[:, 1:]).all() and torch.isfinite(h[:, 0, 0, 1:]).all()
