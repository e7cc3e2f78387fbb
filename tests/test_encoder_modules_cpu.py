"""The encoder's modules and functions around their launches: casts, caches, devices, autograd's other modes (CPU)."""
import pytest
import torch

from paper_2607_21271_amd import rotary
from paper_2607_21271_amd.encoder import EQEncoder, EQWindowBlock


@pytest.mark.parametrize("cast", [lambda m: m.half(), lambda m: m.bfloat16(), lambda m: m.double(), lambda m: m.half().float(),
                                  lambda m: m.to(torch.bfloat16), lambda m: m.to("meta").to_empty(device="cpu")])
def test_frequencies_keep_their_values_under_casts(cast):
    sections = (8, 4, 4)
    want = rotary.axis_frequencies(sections)
    block = cast(EQWindowBlock(2, 64, 2, sections))
    assert block.freqs.dtype == torch.float32 and torch.equal(block.freqs, want)
    assert "freqs" in dict(block.named_buffers()) and "freqs" not in block.state_dict()
    enc = cast(EQEncoder(2, 3, 64, 2, 2, sections))
    assert all(torch.equal(b.freqs, want) for b in enc.blocks)


class Launches:
    """The library's entry points replaced by fills: an output holds `value` where a kernel would have written."""

    def __init__(self, monkeypatch):
        import ctypes

        from paper_2607_21271_amd import _lib, ops
        self.sizes, self.value, self.calls = {}, 3.0, []

        def fill(name, out):
            def launch(*args):
                self.calls.append(name)
                n = self.numel
                (ctypes.c_float * n).from_address(args[out])[:] = [self.value] * n
                return 0
            return launch
        for name, out in (("eqlinear_rotary", 4), ("eqlinear_window_attention", 6), ("eqlinear_group_norm_act", 3)):
            monkeypatch.setattr(_lib, name, fill(name, out))
        monkeypatch.setattr(ops, "_check_dev", lambda *ts: None)
        monkeypatch.setattr(ops, "_stream_of", lambda t: 0)


def operators():
    from paper_2607_21271_amd import attention, norm
    pos, freqs = torch.zeros(5, 1, dtype=torch.int32), torch.ones(2)
    w = torch.ones(3)
    return {"rotary": lambda x: rotary.rotary_axes(x, pos, freqs, (2,)),
            "attention": lambda x: attention.window_attention(x, x, x),
            "packed": lambda x: attention.packed_window_attention(torch.cat((x, x, x), 2), 3),
            "norm": lambda x: norm.group_norm_act(x.view(2, 5, 3, 8), w, w, 1)}


@pytest.mark.parametrize("name", ["rotary", "attention", "packed", "norm"])
def test_forward_mode_is_refused_not_dropped(name, monkeypatch):
    """The operators have no forward-mode derivative: a dual tensor is refused, as the library's layers refuse it, and
    never comes back without its tangent."""
    launches = Launches(monkeypatch)
    launches.numel = 2 * 5 * 3 * 8
    f = operators()[name]
    x = torch.randn(2, 5, 3, 8)
    with torch.no_grad(), torch.autograd.forward_ad.dual_level():
        with pytest.raises((RuntimeError, NotImplementedError)):
            f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        assert (f(x) == 3.0).all()  # others pass


@pytest.mark.parametrize("name", ["rotary", "attention", "packed", "norm"])
def test_a_traced_call_runs_again(name, monkeypatch):
    launches = Launches(monkeypatch)
    launches.numel = 2 * 5 * 3 * 8
    f = operators()[name]
    x = torch.randn(2, 5, 3, 8)
    with torch.no_grad():
        traced = torch.jit.trace(f, x, check_trace=False)
        launches.value, launches.calls = 7.0, []
        assert (traced(x) == 7.0).all() and launches.calls


def test_turning_in_place_is_refused_where_it_would_be_missed(monkeypatch):
    launches = Launches(monkeypatch)
    launches.numel = 2 * 5 * 3 * 8
    pos, freqs = torch.zeros(5, 1, dtype=torch.int32), torch.ones(2)
    turn = lambda x: rotary.rotary_axes_(x, pos, freqs, (2,))
    x = torch.randn(2, 5, 3, 8)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError):
            turn(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        assert (turn(torch.randn(2, 5, 3, 8)) == 3.0).all()
    with pytest.raises(ValueError):
        torch.jit.trace(turn, x, check_trace=False)
    assert (turn(x) == 3.0).all()


@pytest.mark.parametrize("filled,n", [(4, 1), (3, 2), (5, 1), (-1, 1)])
def test_tokens_past_the_end_of_a_cache_are_refused(filled, n):
    """One token past a full cache would broadcast into an empty slice: dropped, and its attention zeros."""
    block = EQWindowBlock(2, 8, 2, (1,), right=0)
    cache = tuple(torch.zeros(3, 4, 2, 8) for _ in range(2))
    spans = torch.full((2, 3), filled, dtype=torch.int32)
    with pytest.raises(ValueError, match="cache"):
        block.extend(torch.zeros(3, n, 8, 2), torch.zeros(n, 1, dtype=torch.int32), cache, filled, spans[0] + n, spans[1])


def test_packed_attention_with_positions_needs_frequencies():
    from paper_2607_21271_amd import attention
    x = torch.zeros(2, 5, 3, 8)
    with pytest.raises(ValueError, match="freqs"):
        attention.packed_window_attention(x, 1, torch.zeros(5, 1, dtype=torch.int32), sections=(2,))


def test_launches_go_to_the_tensors_device(monkeypatch):
    """Tensors of another device than the current one: the call runs on theirs, on its current stream."""
    import contextlib
    from types import SimpleNamespace

    from paper_2607_21271_amd import _lib, ops
    log, current = [], [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], getattr(d, "index", d)
        yield
        current[0] = before
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    monkeypatch.setattr(_lib, "eqlinear_rotary", lambda *a: log.append((current[0], *a)) or 0)
    for index in (0, 1):
        ops._launch("eqlinear_rotary", SimpleNamespace(device=SimpleNamespace(type="cuda", index=index)), 7, 8)
    assert log == [(0, 7, 8, 100), (1, 7, 8, 101)] and current == [0]
    monkeypatch.setattr(_lib, "eqlinear_rotary", lambda *a: _lib.EQL_ERR_INVALID_ARG)
    with pytest.raises(_lib.EqlError):
        ops._launch("eqlinear_rotary", SimpleNamespace(device=SimpleNamespace(type="cuda", index=1)), 7, 8)
