"""What the torch functions of the recurrent operators refuse, before anything runs (CPU), and the recurrent block's
construction."""
import pytest
import torch

from paper_2607_21271_amd import _lib as L, norm, scan
from paper_2607_21271_amd.encoder import EQEncoder, EQScanBlock


def scan_args(B=2, Lt=5, C=6, T=2, N=3, G=2, dt=torch.float16, **kw):
    r = lambda *s: torch.randn(*s).to(dt)
    f = lambda *s: torch.randn(*s)
    a = dict(x=r(B, Lt, C, T), delta=r(B, Lt, C, T), A=f(C, N), Bt=r(B, Lt, G, N), Ct=r(B, Lt, G, N), D=f(C), z=r(B, Lt, C, T),
             delta_bias=f(C), state=f(B, C, T, N))
    a.update(kw)
    return a


h = torch.float16


@pytest.mark.parametrize("kw,error", [
    (dict(x=torch.zeros(2, 5, 12, dtype=h)), ValueError), (dict(delta=torch.zeros(2, 5, 6, 1, dtype=h)), ValueError),
    (dict(z=torch.zeros(2, 4, 6, 2, dtype=h)), ValueError), (dict(A=torch.zeros(5, 3)), ValueError), (dict(A=torch.zeros(6)), ValueError),
    (dict(Bt=torch.zeros(2, 5, 4, 3, dtype=h)), ValueError), (dict(Ct=torch.zeros(2, 5, 1, 3, dtype=h)), ValueError),
    (dict(Bt=torch.zeros(2, 5, 2, 4, dtype=h)), ValueError), (dict(D=torch.zeros(5)), ValueError), (dict(delta_bias=torch.zeros(6, 1)), ValueError),
    (dict(state=torch.zeros(2, 6, 2, 4)), ValueError), (dict(state=torch.zeros(2, 6, 2, 3, dtype=h)), TypeError),
    (dict(A=torch.zeros(6, 3, dtype=h)), TypeError), (dict(D=torch.zeros(6, dtype=torch.float64)), TypeError),
    (dict(delta=torch.zeros(2, 5, 6, 2)), TypeError), (dict(x=torch.zeros(2, 5, 6, 2, dtype=torch.float64)), TypeError),
    (dict(), ValueError)])  # the last: tensors that are not on the GPU
def test_scan_refuses(kw, error):
    with pytest.raises(error):
        scan.selective_scan(**scan_args(**kw))


def conv_args(B=2, Lt=5, C=6, T=2, W=4, dt=torch.float16, **kw):
    r = lambda *s: torch.randn(*s).to(dt)
    a = dict(x=r(B, Lt, C, T), weight=r(C, W), bias=r(C), state=r(B, W - 1, C, T))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,error", [
    (dict(x=torch.zeros(2, 6, 2, dtype=h)), ValueError), (dict(weight=torch.zeros(5, 4, dtype=h)), ValueError),
    (dict(weight=torch.zeros(6, 0, dtype=h)), ValueError), (dict(bias=torch.zeros(4, dtype=h)), ValueError),
    (dict(state=torch.zeros(2, 4, 6, 2, dtype=h)), ValueError), (dict(activation="relu"), ValueError), (dict(activation=None), ValueError),
    (dict(weight=torch.zeros(6, 4)), TypeError), (dict(state=torch.zeros(2, 3, 6, 2)), TypeError), (dict(), ValueError)])
def test_conv_refuses(kw, error):
    with pytest.raises(error):
        scan.causal_conv(**conv_args(**kw))


def res_args(B=2, Lt=5, C=6, T=2, dt=torch.float16, **kw):
    r = lambda *s: torch.randn(*s).to(dt)
    a = dict(x=r(B, Lt, C, T), branch=r(B, Lt, C, T), weight=r(C), bias=r(C), scale=r(C), gate=r(B, C), post_weight=r(C), post_bias=r(C))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,error", [
    (dict(x=torch.zeros(6, 2, dtype=h)), ValueError), (dict(branch=torch.zeros(2, 5, 6, 1, dtype=h)), ValueError),
    (dict(weight=torch.zeros(7, dtype=h)), ValueError), (dict(gate=torch.zeros(6, dtype=h)), ValueError),
    (dict(gate=torch.zeros(1, 6, dtype=h)), ValueError), (dict(post_weight=None), ValueError), (dict(weight=None), ValueError),
    (dict(branch=None), ValueError), (dict(kind="group"), ValueError), (dict(scale=torch.zeros(6)), TypeError),
    (dict(branch=None, scale=None, gate=None, post_weight=None, post_bias=None, weight=None, bias=None), ValueError), (dict(), ValueError)])
def test_residual_refuses(kw, error):
    with pytest.raises(error):
        norm.residual_norm(**res_args(**kw))


def test_lengths_are_checked():
    for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32),
                torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            scan._check_lengths(2, torch.zeros(2), bad)


def test_block_keeps_its_decays_in_full_precision():
    block = EQScanBlock(2, 8, layer_scale=0.1, post_norm=True)
    want = [p.detach().clone() for p in (block.A_log, block.D, block.delta_bias)]
    for cast in (lambda b: b.half(), lambda b: b.to(torch.bfloat16), lambda b: b.float()):
        block = cast(block)
        for p, w in zip((block.A_log, block.D, block.delta_bias), want):
            assert p.dtype == torch.float32 and torch.equal(p, w)
    block = block.half()
    assert block.conv_weight.dtype == block.scale1.dtype == block.post2.weight.dtype == torch.float16
    conv, state = block.new_cache(3)
    assert conv.shape == (3, 3, 16, 2) and conv.dtype == torch.float16 and state.shape == (3, 16, 2, 16) and state.dtype == torch.float32
    assert EQScanBlock(2, 8, device="meta").half().A_log.dtype == torch.float32


def test_encoder_chooses_its_mixer():
    kw = dict(T=2, Cin=2, C=8, heads=2, depth=2, sections=(1, 1), patch=2, registers=1, stem=1, groups=2)
    assert all(type(b) is EQScanBlock for b in EQEncoder(**kw, mixer="scan").blocks)
    assert not any(type(b) is EQScanBlock for b in EQEncoder(**kw).blocks)
    with pytest.raises(ValueError):
        EQEncoder(**kw, mixer="state")


def test_strided_views_are_described():
    """Views of a packed buffer keep their strides; tensors whose tokens are not contiguous are copied."""
    t = torch.zeros(2, 5, 12, 2)
    assert scan._tokens_ready((2, 5, 6, 2), t[:, :, 6:].stride()) and not scan._tokens_ready((2, 5, 6, 2), t[:, :, ::2].stride())
    assert scan._tokens(t[:, :, 6:]).data_ptr() == t[:, :, 6:].data_ptr()
    assert scan._tokens(t[:, :, ::2]).is_contiguous()
    assert scan._tokens(t.transpose(0, 1)).stride() == (24, 120, 2, 1)
    assert scan._steps((1, 5, 3), (7, 8, 9), 3) == (0, 8, 9)


class Launches:
    """The library's entry points replaced by fills: each output that is not NULL holds 3 where a kernel would have written."""

    def __init__(self, monkeypatch, n):
        import ctypes

        from paper_2607_21271_amd import _lib, ops
        self.calls = []

        def fill(name, outs):
            def launch(*args):
                self.calls.append(name)
                for o in outs:
                    if args[o]:
                        (ctypes.c_float * n).from_address(args[o])[:] = [3.0] * n
                return 0
            return launch
        for name, outs in (("eqlinear_selective_scan", (11,)), ("eqlinear_causal_conv", (6,)), ("eqlinear_residual_norm", (9, 10))):
            monkeypatch.setattr(_lib, name, fill(name, outs))
        monkeypatch.setattr(ops, "_check_dev", lambda *ts: None)
        monkeypatch.setattr(ops, "_stream_of", lambda t: 0)


def operators():
    A, w = -torch.ones(3, 4), torch.ones(3)
    bc = torch.ones(2, 5, 1, 4)
    return {"scan": lambda x: scan.selective_scan(x, x, A, bc, bc), "conv": lambda x: scan.causal_conv(x, torch.ones(3, 4)),
            "norm": lambda x: norm.residual_norm(x, x, w)[1], "norm alone": lambda x: norm.residual_norm(x, weight=w)[1]}


@pytest.mark.parametrize("name", list(operators()))
def test_forward_mode_is_refused_not_dropped(name, monkeypatch):
    """No forward-mode derivative: a dual tensor is refused and never comes back without its tangent."""
    launches = Launches(monkeypatch, 2 * 5 * 3 * 8)
    f, x = operators()[name], torch.randn(2, 5, 3, 8)
    with torch.no_grad(), torch.autograd.forward_ad.dual_level():
        with pytest.raises((RuntimeError, NotImplementedError)):
            f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        assert (f(x) == 3.0).all() and launches.calls


@pytest.mark.parametrize("name", list(operators()))
def test_a_traced_call_runs_again(name, monkeypatch):
    launches = Launches(monkeypatch, 2 * 5 * 3 * 8)
    f, x = operators()[name], torch.randn(2, 5, 3, 8)
    with torch.no_grad():
        traced = torch.jit.trace(f, x, check_trace=False)
        launches.calls = []
        assert (traced(x) == 3.0).all() and launches.calls


def test_a_state_in_place_is_not_traced_or_transformed(monkeypatch):
    Launches(monkeypatch, 1)
    state = torch.zeros(2, 3, 3, 8)
    f = lambda x: scan.causal_conv(x, torch.ones(3, 4), state=state, state_out=state)[0]
    x = torch.randn(2, 5, 3, 8)
    with torch.no_grad(), pytest.raises(ValueError):
        torch.jit.trace(f, x, check_trace=False)
    with pytest.raises(ValueError):
        f(x.requires_grad_())
    with torch.no_grad():
        before = state._version
        f(x)
    assert state._version > before
