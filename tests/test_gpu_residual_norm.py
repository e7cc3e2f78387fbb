"""The residual sum between two norms on the GPU against its 64-bit definition (tests/recurrent_ref.py)."""
import itertools

import pytest
import torch

import recurrent_ref as R
from encoder_ref import DT

pytestmark = pytest.mark.gpu

NAMES = ("x", "branch", "weight", "bias", "scale", "gate", "post_weight", "post_bias")


def make(seed, B, L, C, T, dt, weight=True, bias=True, scale=True, gate=True, post=True, post_bias=True, branch=True):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g).to(DT[dt]).cuda()
    t = dict(x=n(B, L, C, T) + 0.5, branch=n(B, L, C, T), weight=n(C), bias=n(C), scale=n(C), gate=n(B, C), post_weight=n(C), post_bias=n(C))
    drop = [k for k, on in (("weight", weight), ("bias", bias and weight), ("scale", scale), ("gate", gate), ("post_weight", post),
                            ("post_bias", post and post_bias), ("branch", branch)) if not on]
    if not branch:
        drop += ["scale", "gate", "post_weight", "post_bias"]
    return {k: None if k in drop else v for k, v in t.items()}


def run(t, dr=None, dh=None, **kw):
    from paper_2607_21271_amd.norm import residual_norm
    if dr is None and dh is None:
        with torch.no_grad():
            r, h = residual_norm(**t, **kw)
        return {k: v for k, v in (("r", r), ("h", h)) if v is not None}
    t = {k: None if v is None else v.detach().requires_grad_() for k, v in t.items()}
    r, h = residual_norm(**t, **kw)
    outs, given = zip(*((o, g) for o, g in ((r, dr), (h, dh)) if g is not None))
    want = [k for k in NAMES if t[k] is not None]
    grads = torch.autograd.grad(outs, [t[k] for k in want], given, allow_unused=True)
    return {**{k: v for k, v in (("r", r), ("h", h)) if v is not None}, **{"d" + k: g for k, g in zip(want, grads) if g is not None}}


def check(t, dr=None, dh=None, **kw):
    shape = t["x"].shape
    flat = lambda v: None if v is None else v.reshape(shape[0], -1, *shape[-2:]) if v.shape == shape else v
    got = run(t, dr, dh, **kw)
    want = R.residual(**{k: flat(v) for k, v in t.items()}, dr=flat(dr), dh=flat(dh), **kw)
    for n, v in got.items():
        if n in want:
            R.within(n, flat(v), *want[n])
    return got


def grads(seed, t):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(t["x"].shape, generator=g).to(t["x"].dtype).cuda() for _ in range(2))


# rows of one element up to the largest, on and off whole vectors, of every number of threads a row
ROWS = [(2, 3, 1, 1), (3, 5, 5, 3), (2, 9, 16, 8), (1, 7, 130, 1), (2, 40, 96, 8), (1, 5, 115, 3), (2, 6, 129, 8), (1, 4, 1025, 2), (2, 3, 4096, 1),
        (1, 3, 1024, 8), (1, 2, 8191, 1), (2, 1, 520, 8), (3, 70, 9, 1), (2, 40, 11, 5), (2, 70, 67, 3), (1, 2, 8192, 1), (2, 3, 1365, 3), (1, 700, 2, 3),
        (2, 33, 16, 1), (1, 9, 40, 2), (2, 9, 50, 4), (3, 5, 100, 5), (1, 8, 400, 2), (1, 3, 300, 4), (2, 3, 620, 4), (2, 5, 1030, 4)]


@pytest.mark.parametrize("size", ROWS, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows(size, dt, kind):
    if kind == "layer" and size[2] * size[3] == 1:
        kind = "rms"  # the mean of one element leaves nothing to normalise
    t = make(sum(size), *size, dt)
    check(t, kind=kind)
    check(t, *grads(3, t), kind=kind)


OPTIONS = [dict(zip(("weight", "bias", "scale", "gate", "post", "post_bias"), c)) for c in itertools.product([0, 1], repeat=6)
           if (c[0] or not c[1]) and (c[4] or not c[5])]


@pytest.mark.parametrize("option", OPTIONS, ids=lambda o: "".join(str(v) for v in o.values()))
@pytest.mark.parametrize("C", [12, 11])
def test_what_may_be_left_out(option, C):
    t = make(5, 3, 20, C, 4, "f16", **option)
    dr, dh = grads(4, t)
    check(t)
    check(t, dr, None)
    if option["weight"]:
        check(t, dr, dh)
        check(t, None, dh)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("bias", [0, 1])
def test_without_a_branch(kind, bias):
    from paper_2607_21271_amd.norm import residual_norm
    t = make(6, 2, 30, 12, 4, "bf16", branch=False, bias=bias)
    check(t, kind=kind)
    check(t, None, grads(5, t)[1], kind=kind)
    r, _ = residual_norm(**t, kind=kind)
    assert r is t["x"]


@pytest.mark.parametrize("B,L", [(1, 5000), (700, 3), (3, 1111)])
@pytest.mark.parametrize("gate", [0, 1])
def test_many_rows(B, L, gate):
    t = make(7, B, L, 10, 4, "f32", gate=gate)
    check(t, *grads(6, t))


def test_other_shapes_and_layouts():
    """Axes between sequence and channel; rows that are not dense; an address off 16 bytes; a broadcast gradient."""
    from paper_2607_21271_amd.norm import residual_norm
    t = make(8, 2, 12, 8, 4, "f16")
    t["x"], t["branch"] = t["x"].view(2, 3, 4, 8, 4), t["branch"].view(2, 3, 4, 8, 4)
    g = tuple(v.view(2, 3, 4, 8, 4) for v in grads(7, t))
    first = check(t, *g)
    u = dict(t, x=torch.cat((t["x"], t["x"]), 3)[..., :8, :], branch=t["branch"].transpose(1, 2).contiguous().transpose(1, 2))
    flat = torch.empty(t["x"].numel() + 1, dtype=torch.float16, device="cuda")
    flat[1:] = t["x"].reshape(-1)
    w = dict(t, x=flat[1:].view(t["x"].shape))
    for other in (u, w):
        for k, v in check(other, *g).items():
            assert v.shape == first[k].shape, k
    x = t["x"].detach().requires_grad_()
    r, h = residual_norm(**dict(t, x=x))
    (r.sum() + h.sum()).backward()
    one = torch.ones(2, 12, 8, 4).half()
    flat4 = {k: v.view(2, 12, 8, 4) if v.dim() == 5 else v for k, v in t.items()}
    R.within("dx", x.grad.view(2, 12, 8, 4), *R.residual(**flat4, dr=one, dh=one)["dx"])


@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_far_values(dt):
    """A mean of 300 beside deviations of one: two passes keep the variance's digits."""
    t = make(9, 2, 20, 24, 4, dt)
    t["x"] = t["x"] + 300
    t["branch"] = t["branch"] - 200
    check(t, *grads(8, t))


def test_dropped_branch():
    """A gate of 0: the branch's gradient is 0, the gate's is not, and a NaN of the branch of another sequence stays there."""
    t = make(10, 3, 20, 12, 4, "f32", post=False)
    t["gate"][1] = 0.0
    got = check(t, *grads(9, t))
    assert (got["dbranch"][1] == 0).all() and (got["dgate"][1] != 0).any()
    t["branch"][0] = float("nan")
    with torch.no_grad():
        got = run(t)
    assert torch.isnan(got["r"][0]).all() and torch.isfinite(got["r"][1:]).all() and torch.isfinite(got["h"][1:]).all()


def test_empty():
    for B, L in ((0, 5), (2, 0)):
        t = make(11, B, L, 4, 2, "f32")
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (4, 4, 4, 4, 4, 4, 8, 8)]
        del junk  # what is allocated next holds NaN
        got = run(t, *grads(1, t))
        assert got["r"].shape == (B, L, 4, 2) and all((got["d" + k] == 0).all() for k in NAMES[2:])


def test_same_bits_every_time():
    t = make(12, 4, 500, 24, 4, "bf16")
    g = grads(2, t)
    first = run(t, *g)
    for _ in range(3):
        for k, v in run(t, *g).items():
            assert torch.equal(v, first[k]), k


def test_branch_is_x():
    from paper_2607_21271_amd.norm import residual_norm
    t = make(14, 2, 9, 12, 4, "f32")
    dr, dh = grads(5, t)
    want = R.residual(**{**t, "branch": t["x"]}, dr=dr, dh=dh)
    x = t["x"].detach().requires_grad_()
    r, h = residual_norm(**{**t, "x": x, "branch": x})
    torch.autograd.backward((r, h), (dr, dh))
    R.within("r", r.detach(), *want["r"])
    R.within("h", h.detach(), *want["h"])
    # a sum of two rounded gradients: its own rounding, half a step of f32, beside their bounds
    both = want["dx"][0] + want["dbranch"][0]
    R.within("dx", x.grad, both, want["dx"][1] + want["dbranch"][1] + both.abs() * 2.0 ** -24 + 2.0 ** -126)


def test_more_sequences_than_a_launch_takes():
    """17 million sequences with gates of their own: workgroups are numbered from each launch's first sequence."""
    B, C = 17_000_003, 8
    t = make(15, 5, 1, C, 1, "f16", bias=False, post=False)
    many = {k: v if v is None or v.shape[0] != 5 else v.repeat(B // 5 + 1, *[1] * (v.dim() - 1))[:B] for k, v in t.items()}
    dr, dh = grads(6, t)
    got, want = run(many), run(t)
    for k in ("r", "h"):
        assert torch.equal(got[k], want[k].repeat(B // 5 + 1, 1, 1, 1)[:B]), k
    more = lambda v: v.repeat(B // 5 + 1, 1, 1, 1)[:B]
    got, want = run(many, more(dr), more(dh)), run(t, dr, dh)
    for k in ("dx", "dbranch", "dgate"):
        assert torch.equal(got[k], want[k].repeat(B // 5 + 1, *[1] * (want[k].dim() - 1))[:B]), k
