"""Group norm with an activation over batches of more workgroups than one launch holds: sequences on either side of a
slice's end give what they give alone, weights and biases the gradients of all of them."""
import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu


def random(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=torch.float16)


# B, S, C, groups (T = 1), sequences of a slice: groups of one channel in passes (one launch); held groups; passes
@pytest.mark.parametrize("B,S,C,G,cut", [(262144, 16, 32, 32, 262143), ((1 << 18) + 5, 1, 512, 64, (1 << 24) // 64),
                                         (16400, 1, 65532, 12, 16367)])
def test_gradients(B, S, C, G, cut):
    from paper_2607_21271_amd.norm import group_norm_act
    x, dy = random(1, B, S, C, 1).requires_grad_(), random(2, B, S, C, 1)
    w, b = (random(3 + i, C).mul_(0.3).add_(s).requires_grad_() for i, s in enumerate((1.0, 0.0)))
    y = group_norm_act(x, w, b, G, "none")
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)
    at = sorted({0, 1, cut - 1, min(cut, B - 1), min(cut + 1, B - 1), B - 1})
    few = x.detach()[at].requires_grad_()
    y_few = group_norm_act(few, w, b, G, "none")
    assert torch.equal(y[at], y_few)
    assert torch.equal(dx[at], torch.autograd.grad(y_few, few, dy[at])[0])
    sums = torch.zeros(4, C, dtype=torch.float64, device="cuda")
    for i in range(0, B, max(1, (1 << 25) // (S * C))):
        part = slice(i, i + max(1, (1 << 25) // (S * C)))
        v = x.detach()[part].double().view(-1, S, G, C // G)
        v = v - v.mean((1, 3), keepdim=True)
        xh = (v * torch.rsqrt(v.pow(2).mean((1, 3), keepdim=True) + 1e-5)).view(-1, C)
        g = dy[part].double().view(-1, C)
        sums += torch.stack(((g * xh).sum(0), g.sum(0), (g.abs() * (1 + xh.abs())).sum(0), g.abs().sum(0)))
    want_w, want_b, size_w, size_b = sums.cpu()
    u = R.U[torch.float16]
    R.within("dw", dw, want_w, u * want_w.abs() + R.E32 * size_w + R.TINY[torch.float16])
    R.within("db", db, want_b, u * want_b.abs() + R.E32 * size_b + R.TINY[torch.float16])


def test_forward_in_passes():
    from paper_2607_21271_amd.norm import group_norm_act
    B, C = 65600, 65532
    x, w, b = random(5, B, 1, C, 1), random(6, C), random(7, C)
    with torch.no_grad():
        y = group_norm_act(x, w, b, 12, "none")
        at = [0, 65534, 65535, 65536, B - 1]
        assert torch.equal(y[at], group_norm_act(x[at], w, b, 12, "none"))
