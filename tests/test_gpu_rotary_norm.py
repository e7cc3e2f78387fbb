"""Rotary positions and group norm with an activation against their definitions in 64 bits (tests/encoder_ref.py)."""
import math

import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu
DT = R.DT


def draw(seed, dt, *shape, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale + shift).to(DT[dt]).cuda()


# ---- rotary ---------------------------------------------------------------------------------------------------------

# B, L, heads, dh, T, sections, interleaved
ROTARY = [
    (1, 1, 1, 2, 1, (1,), False), (1, 1, 1, 2, 1, (1,), True),
    (2, 7, 3, 64, 1, (32,), False), (2, 7, 3, 64, 1, (32,), True),
    (2, 65, 4, 8, 8, (2, 1, 1), False), (2, 65, 4, 8, 8, (2, 1, 1), True),
    (1, 33, 5, 48, 1, (8, 8, 8), False), (1, 130, 2, 10, 3, (2, 1), False), (1, 130, 2, 10, 3, (2, 1), True),
    (3, 9, 2, 16, 4, (3,), True), (3, 9, 2, 16, 4, (0, 3, 2), False), (1, 20, 33, 5, 1, (1, 1), True),
    (2, 40, 1, 512, 2, (100, 100, 56), False), (1, 5, 2, 7, 16, (1, 1, 1), False),
]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_rotary_and_gradient(case, dt):
    from paper_2607_21271_amd.rotary import axis_frequencies, rotary_axes, rotary_axes_
    B, L, N, dh, T, sections, il = case
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-50, 5000, (B, L, len(sections)), generator=g, dtype=torch.int32).cuda()
    freqs = axis_frequencies(sections, device="cuda")
    x = draw(1, dt, B, L, N, dh * T).requires_grad_()
    y = rotary_axes(x, pos, freqs, sections, T, il)
    R.within("y", y, *R.rotary(x, pos, freqs, sections, T, il))
    dy = draw(2, dt, B, L, N, dh * T)
    (dx,) = torch.autograd.grad(y, (x,), dy)
    R.within("dx", dx, *R.rotary(dy, pos, freqs, sections, T, il, inverse=True))
    packed = draw(4, dt, B, L, N + 2, dh * T)  # a view, and in place on it
    keep = packed.clone()
    want = rotary_axes(keep[:, :, 1:N + 1].contiguous(), pos, freqs, sections, T, il)
    assert torch.equal(rotary_axes(packed[:, :, 1:N + 1], pos, freqs, sections, T, il), want)
    rotary_axes_(packed[:, :, 1:N + 1], pos, freqs, sections, T, il)
    assert torch.equal(packed[:, :, 1:N + 1], want)
    assert torch.equal(packed[:, :, 0], keep[:, :, 0]) and torch.equal(packed[:, :, N + 1], keep[:, :, N + 1])
    shared = rotary_axes(x.detach(), pos[0], freqs, sections, T, il)  # positions shared by the batch
    assert torch.equal(shared, rotary_axes(x.detach(), pos[:1].expand(B, L, len(sections)), freqs, sections, T, il))


def test_rotary_far_positions_and_float_positions():
    from paper_2607_21271_amd.rotary import axis_frequencies, rotary_axes
    freqs = axis_frequencies((16, 16), device="cuda")
    pos = torch.tensor([[0, 0], [1, 2], [1 << 20, 3], [(1 << 24) - 1, -(1 << 24)]], dtype=torch.int32, device="cuda")
    x = draw(5, "f32", 1, 4, 2, 64)
    y = rotary_axes(x, pos, freqs, (16, 16))
    R.within("int", y, *R.rotary(x, pos, freqs, (16, 16), 1, False))
    assert torch.equal(y[:, 0], x[:, 0])  # the origin does not turn
    assert torch.equal(y, rotary_axes(x, pos.float(), freqs, (16, 16)))
    half = pos.float() * 0.37 + 0.1
    R.within("float", rotary_axes(x, half, freqs, (16, 16)), *R.rotary(x, half, freqs, (16, 16), 1, False))


def test_rotary_commutes_with_the_group_and_other_stream():
    from paper_2607_21271_amd.rotary import axis_frequencies, grid_positions, rotary_axes
    T, dh, N = 8, 8, 3
    pos = grid_positions((3, 4, 5), prefix=2, device="cuda")
    assert pos.shape == (62, 3) and pos[2:].tolist()[7] == [0, 1, 2] and pos[:2].abs().sum() == 0
    freqs = axis_frequencies((2, 1, 1), theta=(1e4, 100.0, 100.0), device="cuda")
    x = draw(6, "f16", 2, 62, N, dh * T)
    roll = lambda t: t.view(2, 62, N, dh, T).roll(3, -1).reshape(2, 62, N, dh * T)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = rotary_axes(roll(x), pos, freqs, (2, 1, 1), T)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, roll(rotary_axes(x, pos, freqs, (2, 1, 1), T)))


# ---- group norm -----------------------------------------------------------------------------------------------------

# B, S, C, T, groups
NORM = [(1, 1, 8, 4, 1), (2, 3, 24, 4, 4), (1, 196, 24, 4, 6), (3, 50, 5, 3, 5), (2, 64, 64, 4, 16), (1, 7, 300, 8, 10),
        (2, 17, 1030, 2, 103), (5, 129, 16, 1, 2), (1, 2000, 12, 2, 3), (70, 9, 8, 2, 2),
        (2, 300, 24, 4, 4), (1, 1500, 16, 8, 2), (1, 5300, 24, 4, 4), (3, 700, 64, 4, 1), (1, 21000, 8, 2, 2)]


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", NORM, ids=lambda c: "x".join(map(str, c)))
def test_group_norm_and_gradients(case, dt, act):
    from paper_2607_21271_amd.norm import group_norm_act
    B, S, C, T, G = case
    x = draw(11, dt, B, S, C, T, scale=1.5, shift=0.7).requires_grad_()
    w, b = draw(12, dt, C, scale=0.3, shift=1.0).requires_grad_(), draw(13, dt, C, scale=0.3).requires_grad_()
    dy = draw(14, dt, B, S, C, T)
    y = group_norm_act(x, w, b, G, act, eps=1e-5)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)
    want = R.group_norm_act(x, w, b, G, act, 1e-5, dy)
    got = {"y": y, "dx": dx, "dw": dw, "db": db}
    if act == "relu":
        # a value within rounding of zero may fall on either side: its derivative is not compared
        z = R.group_norm_act(x, w, b, G, "none", 1e-5)["y"][0]
        near = z.abs() < 1e-4
        want["dx"] = (want["dx"][0], torch.where(near, math.inf, want["dx"][1]))
        slack = (near.double() * dy.double().cpu().abs() * 8).sum((0, 1, 3))
        want["dw"], want["db"] = ((v, e + slack) for v, e in (want["dw"], want["db"]))
        want["dx"] = (want["dx"][0], want["dx"][1] + near.any().double() * 1e-2)
    for n, t in got.items():
        R.within(n, t, *want[n])
    with torch.no_grad():
        assert torch.equal(group_norm_act(x, w, b, G, act, eps=1e-5), y)


@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_group_norm_far_mean_and_constant_groups(dt):
    """A mean 300 spreads from zero does not cancel; a group of equal values gives bias."""
    from paper_2607_21271_amd.norm import group_norm_act
    x = draw(21, dt, 2, 100, 8, 2, scale=1.0, shift=300.0)
    w, b = draw(22, dt, 8, shift=1.0), draw(23, dt, 8)
    R.within("far", group_norm_act(x, w, b, 2), *R.group_norm_act(x, w, b, 2, "none", 1e-5)["y"])
    x[:, :, :4] = 3.25
    y = group_norm_act(x, w, b, 2)
    assert torch.equal(y[:, :, :4], b[:4, None].expand(2, 100, 4, 2))


def test_group_norm_shapes_streams_graph_and_group():
    from paper_2607_21271_amd.norm import GroupNormAct, group_norm_act
    m = GroupNormAct(16, 4, "silu", device="cuda", dtype=torch.float16)
    with torch.no_grad():
        m.weight.copy_(draw(31, "f16", 16, shift=1.0))
        m.bias.copy_(draw(32, "f16", 16))
    x = draw(33, "f16", 2, 9, 11, 16, 4)
    with torch.no_grad():
        y = m(x)
        assert y.shape == x.shape and torch.equal(y.view(2, 99, 16, 4), m(x.view(2, 99, 16, 4)))
        assert torch.equal(m(x.permute(0, 2, 1, 3, 4)), group_norm_act(x.permute(0, 2, 1, 3, 4).contiguous(), m.weight, m.bias, 4, "silu"))
        R.within("roll", m(x.roll(1, -1)), *((t.roll(1, -1)) for t in R.group_norm_act(x, m.weight, m.bias, 4, "silu", 1e-5)["y"]))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            z = m(x)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(z, y)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = m(x)
        for step in range(3):
            x.copy_(draw(40 + step, "f16", 2, 9, 11, 16, 4))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, m(x)), step
    e = torch.zeros(0, 5, 16, 4, dtype=torch.float16, device="cuda", requires_grad=True)
    assert m(e).shape == e.shape
    dx, dw, _ = torch.autograd.grad(m(e).sum(), (e, m.weight, m.bias))
    assert dx.shape == e.shape and (dw == 0).all()


def test_group_norm_gradient_against_differences():
    from paper_2607_21271_amd.norm import group_norm_act
    x, w, b = draw(51, "f32", 2, 30, 6, 2), draw(52, "f32", 6, shift=1.0), draw(53, "f32", 6)
    dy = draw(54, "f32", 2, 30, 6, 2)
    t = [v.clone().requires_grad_() for v in (x, w, b)]
    grads = torch.autograd.grad(group_norm_act(*t, 3, "gelu"), t, dy)
    h = 1e-2
    for i in range(3):
        d = draw(60 + i, "f32", *t[i].shape)
        f = []
        for s in (h, -h):
            v = [x, w, b]
            v[i] = v[i] + s * d
            f.append((group_norm_act(*v, 3, "gelu").double() * dy.double()).sum())
        diff, dot = ((f[0] - f[1]) / (2 * h)).item(), (grads[i].double() * d.double()).sum().item()
        size = (grads[i].double().abs() * d.double().abs()).sum().item()
        # h^2 / 6 of third derivatives a few times the first, 2^-22 / h of the outputs
        assert abs(diff - dot) <= (4 * h * h + 2.0 ** -22 / h) * size + 1e-2, (i, diff, dot)
