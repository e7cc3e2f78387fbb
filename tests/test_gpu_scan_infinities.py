"""The selective scan with infinities inside its sequences, on the GPU, against its 64-bit definition: what is infinite there is
infinite with the same sign, what is NaN there is NaN, everything else is within the bounds of tests/recurrent_ref.py.  Of
gradients, those that are infinite or NaN there are infinite or NaN."""
import pytest
import torch

import recurrent_ref as R
from encoder_ref import DT
from test_gpu_scan import run

pytestmark = pytest.mark.gpu
INF = float("inf")


def positive(seed, B, L, C, T, N, G, dt):
    """Everything but A is positive, so that an infinity keeps its sign, and the decays are far from the least normal numbers."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: (torch.rand(*s, generator=g) + 0.25)
    e = lambda t: t.to(DT[dt]).cuda()
    return dict(x=e(n(B, L, C, T)), delta=e(n(B, L, C, T)), A=-n(C, N).cuda() / 2, Bt=e(n(B, L, G, N)), Ct=e(n(B, L, G, N)), D=n(C).cuda(),
                z=e(n(B, L, C, T)), delta_bias=n(C).cuda() - 4, state=n(B, C, T, N).cuda())


def same(name, got, want, bound):
    got, fin = got.double().cpu(), torch.isfinite(want)
    if name in ("y", "state"):
        assert (torch.isnan(got) == torch.isnan(want)).all(), "%s: NaN %d, expected %d" % (name, torch.isnan(got).sum(), torch.isnan(want).sum())
        off = ~fin & ~torch.isnan(want)
        assert torch.equal(got[off], want[off]), name
    assert torch.equal(torch.isfinite(got), fin), name
    known = fin & torch.isfinite(bound)
    assert ((got - want).abs()[known] <= bound[known]).all(), name


def check(t, dy=None, ds=None, **kw):
    got, want = run(t, dy, ds, **kw), R.scan(**t, dy=dy, dstate=ds, **kw)
    for k, v in got.items():
        if k in want:
            same(k, v, *want[k])
    return got


# every number of lanes that share columns with states short of whole runs and of whole lanes (and none short); rows of whole
# vectors, of vectors that end with the group, and shorter than a vector; few tokens, tiles, chunks
STATES = [1, 2, 3, 4, 5, 7, 12, 15, 20, 31, 40, 62]


@pytest.mark.parametrize("N", STATES)
@pytest.mark.parametrize("C", [16, 33, 3])
@pytest.mark.parametrize("L", [3, 40, 700])
@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_infinite_elements(N, C, L, dt):
    """One infinite element of x, in one column: y is infinite from its token on there, and nowhere else."""
    t = positive(N + C, 2, L, C, 1, N, 1, dt)
    t["x"][0, L // 2, C // 2] = INF
    t["x"][1, 1, C - 1] = -INF
    got = check(t)
    assert torch.isinf(got["y"][0, L // 2:, C // 2]).all() and torch.isfinite(got["y"][0, :, :C // 2]).all()


@pytest.mark.parametrize("N", [1, 7, 12, 33, 64])
def test_infinite_steps(N):
    """An infinite step forgets the state (exp of -inf) and adds an infinity."""
    t = positive(N, 1, 40, 5, 3, N, 1, "f32")
    t["delta"][0, 20, 2, 1] = INF
    check(t)
    g = torch.Generator().manual_seed(5)
    check(t, torch.rand(1, 40, 5, 3, generator=g).cuda() + 0.25)


@pytest.mark.parametrize("N", STATES + [64])
@pytest.mark.parametrize("C", [16, 33, 3])
@pytest.mark.parametrize("L", [20, 300])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_infinite_gradients(N, C, L, dt):
    """One infinite element of dy."""
    t = positive(N + C + 1, 2, L, C, 1, N, 1, dt)
    g = torch.Generator().manual_seed(3)
    dy = (torch.rand(2, L, C, 1, generator=g) + 0.25).to(t["x"].dtype).cuda()
    dy[0, L // 2, C // 2] = INF
    check(t, dy)


@pytest.mark.parametrize("what", ["x", "Bt", "Ct"])
@pytest.mark.parametrize("N", [3, 12, 16, 64])
@pytest.mark.parametrize("C", [5, 35, 72])
@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_infinities_and_gradients(what, N, C, dt):
    """An infinite element of x, b or c, in groups that leave columns of a wave empty; gradients of y and of the last state."""
    L = 50
    t = positive(N + C + 2, 2, L, C, 1, N, 1, dt)
    t[what][1, 17, 0, 0] = INF
    g = torch.Generator().manual_seed(4)
    p = lambda *s: torch.rand(*s, generator=g).cuda() + 0.25
    check(t, p(2, L, C, 1).to(t["x"].dtype), p(2, C, 1, N))
