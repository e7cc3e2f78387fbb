"""The 64-bit references of the recurrent operators: their gradients against central differences of their values, and a
mistake planted in each is caught by the bounds (CPU)."""
import pytest
import torch

import recurrent_ref as ref

torch.manual_seed(3)


def rnd(*shape, scale=1.0):
    return torch.randn(*shape, dtype=torch.float64) * scale


def differences(f, t, given, step=1e-5):
    """d sum(f * given) / dt by central differences."""
    out = torch.zeros_like(t)
    flat, o = t.reshape(-1), out.reshape(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        vals = []
        for s in (step, -step):
            flat[i] = keep + s
            vals.append(sum((a * b).sum() for a, b in zip(f(), given)))
        flat[i] = keep
        o[i] = (vals[0] - vals[1]) / (2 * step)
    return out


def near(name, got, want):
    if want.numel() == 0:
        return
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-7 * (1 + want.abs().max().item())), (name, got, want)


@pytest.fixture(autouse=True)
def exact_types(monkeypatch):
    """64-bit inputs: no rounding of results."""
    monkeypatch.setitem(ref.U, torch.float64, 0.0)
    monkeypatch.setitem(ref.TINY, torch.float64, 0.0)


@pytest.mark.parametrize("softplus", [True, False])
def test_scan_gradients(softplus):
    B, L, C, T, N, G = 2, 4, 4, 2, 3, 2
    t = dict(x=rnd(B, L, C, T), delta=rnd(B, L, C, T, scale=0.3) + (0 if softplus else 0.5), A=-torch.rand(C, N, dtype=torch.float64),
             Bt=rnd(B, L, G, N), Ct=rnd(B, L, G, N), D=rnd(C), z=rnd(B, L, C, T), delta_bias=rnd(C, scale=0.2),
             state=rnd(B, C, T, N))
    lengths = torch.tensor([4, 3])
    gy, gs = rnd(B, L, C, T), rnd(B, C, T, N)
    out = ref.scan(**t, softplus=softplus, lengths=lengths, dy=gy, dstate=gs)

    def f():
        o = ref.scan(**t, softplus=softplus, lengths=lengths)
        return o["y"][0], o["state"][0]

    for name, key in (("x", "dx"), ("delta", "ddelta"), ("A", "dA"), ("Bt", "dBt"), ("Ct", "dCt"), ("D", "dD"), ("z", "dz"),
                      ("delta_bias", "dbias"), ("state", "dstate")):
        near(name, out[key][0], differences(f, t[name], (gy, gs)))


@pytest.mark.parametrize("activation", ["none", "silu"])
@pytest.mark.parametrize("W", [1, 2, 4])
def test_conv_gradients(activation, W):
    B, L, C, T = 2, 3, 3, 2
    t = dict(x=rnd(B, L, C, T), weight=rnd(C, W), bias=rnd(C), state=rnd(B, W - 1, C, T))
    lengths = torch.tensor([3, 1])
    gy, gs = rnd(B, L, C, T), rnd(B, W - 1, C, T)
    out = ref.conv(**t, activation=activation, lengths=lengths, dy=gy, dstate=gs)

    def f():
        o = ref.conv(**t, activation=activation, lengths=lengths)
        return o["y"][0], o["state"][0]

    for name, key in (("x", "dx"), ("weight", "dw"), ("bias", "db"), ("state", "dstate")):
        near(name, out[key][0], differences(f, t[name], (gy, gs)))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
def test_residual_gradients(kind, post):
    B, L, C, T = 2, 2, 4, 2
    t = dict(x=rnd(B, L, C, T), branch=rnd(B, L, C, T), weight=rnd(C), bias=rnd(C), scale=rnd(C), gate=rnd(B, C))
    if post:
        t |= dict(post_weight=rnd(C), post_bias=rnd(C))
    gr, gh = rnd(B, L, C, T), rnd(B, L, C, T)
    out = ref.residual(**t, kind=kind, eps=1e-3, dr=gr, dh=gh)

    def f():
        o = ref.residual(**t, kind=kind, eps=1e-3)
        return o["r"][0], o["h"][0]

    for name in t:
        near(name, out["d" + name][0], differences(f, t[name], (gr, gh)))


def test_bounds_catch_mistakes():
    """A bound is worth something only where a plausible mistake leaves it: each of these does, for many values."""
    B, L, C, T, N = 1, 40, 3, 2, 4
    t = dict(x=rnd(B, L, C, T).float(), delta=rnd(B, L, C, T).float(), A=-torch.rand(C, N) - 0.2, Bt=rnd(B, L, 1, N).float(),
             Ct=rnd(B, L, 1, N).float(), D=rnd(C).float(), z=rnd(B, L, C, T).float(), delta_bias=rnd(C).float() - 2)
    gy = rnd(B, L, C, T).float()
    out = ref.scan(**t, dy=gy)
    for name, change in (("y", dict(softplus=False)), ("y", dict(A=t["A"] * 1.01)), ("dA", dict(D=None, x=t["x"] * 1.01)),
                         ("ddelta", dict(Bt=t["Bt"].roll(1, 1))), ("dBt", dict(Ct=t["Ct"] * 1.01)),
                         ("dx", dict(delta_bias=None)), ("dz", dict(D=None)), ("dCt", dict(A=t["A"] * 1.01))):
        wrong = ref.scan(**{**t, **change}, dy=gy)[name][0]
        want, bound = out[name]
        assert ((wrong - want).abs() > bound).double().mean() > 0.3, (name, change.keys())
