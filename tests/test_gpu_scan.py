"""The selective scan on the GPU against its 64-bit definition (tests/recurrent_ref.py)."""
import itertools

import pytest
import torch

import recurrent_ref as R
from encoder_ref import DT

pytestmark = pytest.mark.gpu

NAMES = ("x", "delta", "A", "Bt", "Ct", "D", "z", "delta_bias", "state")
GRADS = ("dx", "ddelta", "dA", "dBt", "dCt", "dD", "dz", "dbias", "dstate")


def make(seed, B, L, C, T, N, G, dt, D=True, z=True, bias=True, state=True, softplus=True):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: torch.randn(*s, generator=g) * scale
    e = lambda t: t.to(DT[dt]).cuda()
    f = lambda t: t.float().cuda()
    return dict(x=e(n(B, L, C, T)), delta=e(n(B, L, C, T, scale=0.5) if softplus else n(B, L, C, T, scale=0.1).abs()),
                A=f(-torch.rand(C, N, generator=g) * N - 0.01), Bt=e(n(B, L, G, N)), Ct=e(n(B, L, G, N)),
                D=f(n(C)) if D else None, z=e(n(B, L, C, T)) if z else None,
                delta_bias=f(n(C) - 3.0 if softplus else n(C, scale=0.1).abs()) if bias else None, state=f(n(B, C, T, N)) if state else None)


def run(t, dy=None, dstate=None, **kw):
    """{name: tensor} of the values and, where gradients are given, of the gradients."""
    from paper_2607_21271_amd.scan import selective_scan
    if dy is None and dstate is None:
        with torch.no_grad():
            y, h = selective_scan(**t, return_state=True, **kw)
        return {"y": y, "state": h}
    t = {k: None if v is None else v.detach().requires_grad_() for k, v in t.items()}
    y, h = selective_scan(**t, return_state=True, **kw)
    outs, given = zip(*((o, g) for o, g in ((y, dy), (h, dstate)) if g is not None))
    want = [k for k in NAMES if t[k] is not None]
    # a gradient of the last state alone reaches neither D nor the gate
    grads = torch.autograd.grad(outs, [t[k] for k in want], given, allow_unused=dy is None)
    return {"y": y, "state": h, **{GRADS[NAMES.index(k)]: g for k, g in zip(want, grads)}}


def check(t, dy=None, dstate=None, **kw):
    got, want = run(t, dy, dstate, **kw), R.scan(**t, dy=dy, dstate=dstate, **kw)
    for n, v in got.items():
        if n in want:
            R.within(n, v, *want[n])


def grads(seed, t, L):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(t["x"].shape, generator=g).to(t["x"].dtype).cuda(),
            torch.randn(t["x"].shape[0], *t["A"].shape[:1], t["x"].shape[3], t["A"].shape[1], generator=g).cuda())


# sizes: one token, a tile's edges for every number of lanes that share columns, several column blocks of a group, columns off the
# vectors, chunks of tokens
SIZES = [(1, 1, 1, 1, 1, 1), (2, 1, 8, 4, 16, 1), (3, 5, 6, 1, 4, 2), (2, 17, 12, 8, 16, 1), (1, 16, 3, 5, 7, 3), (2, 33, 40, 8, 16, 2),
         (1, 64, 9, 2, 64, 1), (2, 15, 64, 8, 8, 1), (1, 31, 70, 4, 33, 1), (2, 40, 150, 2, 3, 1), (1, 300, 16, 4, 16, 2), (1, 700, 5, 1, 20, 1),
         (1, 520, 8, 1, 2, 1), (1, 130, 80, 4, 12, 1), (2, 8, 200, 8, 16, 1),
         # a group's last vector not full, in its first block and in a later one; runs of four states not full
         (2, 37, 75, 3, 7, 3), (1, 70, 131, 5, 13, 1), (2, 40, 67, 1, 1, 1), (1, 50, 261, 1, 3, 1), (1, 90, 33, 1, 62, 1), (2, 25, 105, 3, 21, 3),
         (3, 2, 205, 5, 11, 1),
         # few tokens
         (2, 4, 37, 3, 62, 1), (5, 3, 9, 8, 5, 3), (2, 2, 300, 1, 3, 1), (3, 4, 17, 8, 32, 1)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scan(size, dt):
    t = make(sum(size), *size, dt)
    check(t)
    check(t, *grads(5, t, size[1]))


# gradients in workgroups of one, two, three and four waves, several side by side for a group's columns, chunks of several tiles
@pytest.mark.parametrize("size", [(64, 33, 520, 1, 5, 1), (33, 50, 520, 1, 5, 1), (40, 33, 520, 1, 2, 1), (17, 100, 520, 1, 5, 1),
                                  (130, 9, 65, 1, 33, 1), (130, 33, 5, 1, 2, 1), (33, 50, 257, 1, 5, 1), (40, 33, 257, 1, 2, 1),
                                  (17, 100, 257, 1, 5, 1), (130, 9, 257, 1, 5, 1), (40, 50, 129, 1, 2, 1), (1, 33, 97, 1, 16, 1)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_workgroups(size, dt):
    t = make(sum(size), *size, dt)
    lengths = torch.randint(0, size[1] + 1, (size[0],), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    check(t, *grads(5, t, size[1]), lengths=lengths.cuda())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C", [8, 9, 3], ids=["whole", "loose", "tiny"])
@pytest.mark.parametrize("N", [4, 8, 16, 32, 64])
def test_ways_to_read(N, C, dt):
    """Whole vectors, rows that are none, rows shorter than one, for every number of lanes that share columns, two or three tiles
    of one wave."""
    L, n = 10 if N == 4 else 20, N if C == 8 else N - 1
    t = make(N + C, 1030, L, C, 1, n, 1, dt)
    check(t)
    check(t, *grads(7, t, L))
    # without the gate and the softplus
    t = make(N + C, 1030, L, C, 1, n, 1, dt, 1, 0, 1, 0, False)
    check(t, softplus=False)
    check(t, grads(7, t, L)[0], None, softplus=False)


@pytest.mark.parametrize("D,z,bias,state,softplus", [c for c in itertools.product([0, 1], repeat=5) if sum(c) in (0, 1, 4)])
def test_what_may_be_left_out(D, z, bias, state, softplus):
    t = make(7, 2, 21, 8, 4, 16, 1, "bf16", D, z, bias, state, bool(softplus))
    check(t, softplus=bool(softplus))
    check(t, *grads(6, t, 21), softplus=bool(softplus))
    check(t, grads(6, t, 21)[0], None, softplus=bool(softplus))
    check(t, None, grads(6, t, 21)[1], softplus=bool(softplus))


@pytest.mark.parametrize("dt", ["f32", "f16"])
@pytest.mark.parametrize("L", [1, 3, 40, 400])
def test_lengths(dt, L):
    """Sequences of no token, one, all but one, all; what lies behind them is NaN and reaches nothing."""
    lengths = torch.tensor([0, 1, L - 1, L, -3, L + 7], dtype=torch.int32)
    t = make(3, 6, L, 6, 2, 8, 2, dt)
    dy, ds = grads(4, t, L)
    for b, n in enumerate(lengths.clamp(0, L).tolist()):
        for k in ("x", "delta", "Bt", "Ct", "z"):
            t[k][b, n:] = float("nan")
        dy[b, n:] = float("inf")
    check(t, lengths=lengths.cuda())
    got = run(t, dy, ds, lengths=lengths.cuda())
    want = R.scan(**t, dy=dy, dstate=ds, lengths=lengths)
    for n, v in got.items():
        R.within(n, v, *want[n])
    for b, n in enumerate(lengths.clamp(0, L).tolist()):
        for k in ("y", "dx", "ddelta", "dz", "dBt", "dCt"):
            assert (got[k][b, n:] == 0).all(), (k, b)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cut", ["packed", "offset", "odd", "broadcast", "turned"])
def test_layouts(dt, cut):
    """Views of packed buffers, of odd strides and addresses, broadcast over sequences, tokens before sequences."""
    B, L, C, T, N, G = 2, 50, 12, 4, 8, 2
    t = make(11, B, L, C, T, N, G, dt)
    dy, ds = grads(12, t, L)

    def lay(v):
        if v is None or v.dim() != 4:
            return v
        if cut == "packed":
            return torch.cat((v, v + 1), 2)[:, :, :v.shape[2]]
        if cut == "offset":
            flat = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")
            flat[1:] = v.reshape(-1)
            return flat[1:].view(v.shape)
        if cut == "odd":
            wide = torch.zeros(B, L, v.shape[2] * v.shape[3] + 3, dtype=v.dtype, device="cuda")
            wide[:, :, 2:-1] = v.flatten(2)
            return wide[:, :, 2:-1].unflatten(2, v.shape[2:])
        if cut == "broadcast":
            return v[:1].expand(B, *v.shape[1:])
        return v.transpose(0, 1).contiguous().transpose(0, 1)

    state = t.pop("state")
    t = {k: lay(v) for k, v in t.items()}
    t["state"] = state
    check(t, lay(dy), ds)


@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_tokens_far_apart(dt):
    """Tokens 2^24 elements apart, as in a buffer of many sequences side by side."""
    t = make(13, 1, 3, 6, 3, 7, 1, dt)
    dy, ds = grads(14, t, 3)
    wide = torch.zeros(1, 3, (1 << 24) + 5, dtype=t["x"].dtype, device="cuda")
    for i, k in enumerate(("x", "delta", "z", "Bt", "Ct")):
        v = t[k].flatten(2)
        wide[:, :, 100 * i:100 * i + v.shape[2]] = v
        t[k] = wide[:, :, 100 * i:100 * i + v.shape[2]].unflatten(2, t[k].shape[2:])
    check(t)
    check(t, dy, ds)


def test_gradient_of_a_broadcast_sum():
    """y.sum(): a gradient with strides of 0."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(2, 2, 20, 4, 2, 4, 1, "f32", state=False)
    t = {k: None if v is None else v.requires_grad_() for k, v in t.items()}
    selective_scan(**t).sum().backward()
    want = R.scan(**t, dy=torch.ones(2, 20, 4, 2))
    for k, n in zip(NAMES[:-1], GRADS[:-1]):
        R.within(n, t[k].grad, *want[n])


@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_carrying_on(dt):
    """A sequence in pieces of 1, 16, 3 and 300 tokens with the state updated in place, against the whole one."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(21, 2, 320, 8, 4, 16, 2, dt)
    want = R.scan(**t)
    state, at = t["state"].clone(), 0
    version = state._version
    ys = []
    for n in (1, 16, 3, 300):
        part = {k: v[:, at:at + n] if k in ("x", "delta", "Bt", "Ct", "z") else v for k, v in t.items()}
        part["state"] = state
        y, out = selective_scan(**part, state_out=state)
        assert out is state
        ys.append(y)
        at += n
    assert state._version > version
    R.within("y", torch.cat(ys, 1), *want["y"])
    R.within("state", state, *want["state"])


def test_empty():
    t = make(1, 2, 0, 4, 2, 4, 1, "f32")
    got = run(t, torch.zeros_like(t["x"]), torch.ones(2, 4, 2, 4, device="cuda"))
    assert torch.equal(got["state"], t["state"]) and (got["dstate"] == 1).all() and got["y"].shape == (2, 0, 4, 2)
    assert all((got[k] == 0).all() for k in ("dA", "dD", "dbias"))
    t = make(1, 0, 5, 4, 2, 4, 1, "f16")
    got = run(t, torch.zeros_like(t["x"]), torch.ones(0, 4, 2, 4, device="cuda"))
    assert got["y"].shape == (0, 5, 4, 2) and all((got[k] == 0).all() for k in ("dA", "dD", "dbias"))


def test_steep_and_flat_decays():
    """A of 0 (the state keeps everything), of -1e4 (nothing), growing ones, steps of 0 and of 30."""
    t = make(31, 1, 200, 8, 1, 4, 1, "f32", softplus=False)
    t["A"][0], t["A"][1], t["A"][2] = 0.0, -1e4, 0.02
    t["delta_bias"] = None
    t["delta"] = t["delta"].abs()
    t["delta"][:, ::7] = 0.0
    t["delta"][:, 5, 3:] = 30.0
    check(t, *grads(3, t, 200), softplus=False)


def test_long_gradient_of_the_decay():
    """dA over 16 K tokens of one sequence and of 300 short ones: sums keep their digits."""
    for B, L, C, T in ((1, 4096, 4, 1), (300, 24, 4, 4)):
        t = make(41, B, L, C, T, 4, 1, "f32", state=False)
        check(t, grads(8, t, L)[0], None)


def test_same_bits_every_time():
    t = make(51, 2, 600, 24, 4, 16, 1, "f16")
    dy, ds = grads(2, t, 600)
    first = run(t, dy, ds)
    for _ in range(3):
        for k, v in run(t, dy, ds).items():
            assert torch.equal(v, first[k]), k


def test_second_derivative_is_refused():
    from paper_2607_21271_amd.scan import selective_scan
    t = make(2, 1, 4, 4, 2, 4, 1, "f32", state=False)
    x = t["x"].requires_grad_()
    g, = torch.autograd.grad(selective_scan(**t).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)


def test_state_out_is_not_differentiable():
    from paper_2607_21271_amd.scan import selective_scan
    t = make(2, 1, 4, 4, 2, 4, 1, "f32")
    out = torch.empty_like(t["state"])
    t["x"].requires_grad_()
    with pytest.raises(ValueError):
        selective_scan(**t, state_out=out)
    with torch.no_grad():
        y, h = selective_scan(**t, state_out=out)
    assert h is out and not y.requires_grad
    with pytest.raises(ValueError):
        selective_scan(**{k: None if v is None else v.detach() for k, v in t.items()}, state_out=out[:, :2])


@pytest.mark.parametrize("L", [1, 5])
def test_more_waves_than_a_launch_takes(L):
    """4100 sequences of 4096 column blocks: more waves than one launch has, all sequences alike."""
    from paper_2607_21271_amd.scan import selective_scan
    t = make(31, 1, L, 4096, 16, 64, 1, "f16", state=False)
    with torch.no_grad():
        want = selective_scan(**t)
        many = {k: v.expand(4100, *v.shape[1:]) if v is not None and v.dim() == 4 else v for k, v in t.items()}
        got = selective_scan(**many)
    for part in got.split(100):
        assert torch.equal(part, want.expand_as(part))
