"""The recurrent block under autocast: its parts stay of one type, the block's own, and its results are those without."""
import pytest
import torch

from paper_2607_21271_amd import encoder
from paper_2607_21271_amd.encoder import EQEncoder, EQScanBlock


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_one_type_reaches_the_scan(dtype, monkeypatch):
    """Bt and Ct, which come from a dense layer, have the type of x (on the CPU, with the operators replaced)."""
    block = EQScanBlock(2, 8).to(dtype)
    seen = {}

    def scan_(x, delta, A, Bt, Ct, D, z, bias, **kw):
        seen.update(x=x, delta=delta, z=z, Bt=Bt, Ct=Ct, wide=(A, D, bias))
        return x

    monkeypatch.setattr(encoder.EQLinear, "forward", lambda self, x: torch.ones(*x.shape[:-2], self.Cout, self.T, dtype=x.dtype))
    monkeypatch.setattr(encoder.scan, "causal_conv", lambda x, *a, **kw: x)
    monkeypatch.setattr(encoder.scan, "selective_scan", scan_)
    with torch.autocast("cpu", dtype=torch.bfloat16):
        block.mix(torch.ones(1, 3, 8, 2, dtype=dtype))
    assert {k: v.dtype for k, v in seen.items() if k != "wide"} == dict.fromkeys(("x", "delta", "z", "Bt", "Ct"), dtype)
    assert all(t.dtype == torch.float32 for t in seen["wide"])


@pytest.mark.gpu
@pytest.mark.parametrize("own,cast", [(torch.float32, torch.float16), (torch.float32, torch.bfloat16), (torch.float16, torch.bfloat16)])
def test_block_under_autocast(own, cast):
    torch.manual_seed(0)
    block = EQScanBlock(4, 16, layer_scale=0.5, post_norm=True, states=8, groups=2).cuda().to(own)
    x = torch.randn(2, 40, 16, 4, device="cuda").to(own).requires_grad_()
    g = torch.randn(2, 40, 16, 4, device="cuda").to(own)

    def step(on):
        with torch.autocast("cuda", dtype=cast, enabled=on):
            y = block(x)
        return (y, *torch.autograd.grad(y, [x, *block.parameters()], g))

    want, got = step(False), step(True)
    with torch.autocast("cuda", dtype=cast):
        cache = block.new_cache(2)
        parts = [block.extend(x[:, a:b], cache) for a, b in ((0, 1), (1, 40))]
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and torch.equal(a, b)
    cache = block.new_cache(2)
    for p, (a, b) in zip(parts, ((0, 1), (1, 40))):
        assert torch.equal(p, block.extend(x[:, a:b], cache))


@pytest.mark.gpu
def test_encoder_trains_under_autocast():
    torch.manual_seed(1)
    enc = EQEncoder(4, 3, 16, heads=2, depth=2, sections=(1, 1, 1), patch=2, registers=2, stem=1, mixer="scan").cuda()
    x = torch.randn(2, 2, 8, 8, 3, 4, device="cuda")
    with torch.autocast("cuda", dtype=torch.bfloat16):
        loss = enc(x).square().mean()
    loss.backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in enc.parameters())
