"""The encoder on the library's layers: its block against a plain one, training, equivariance, streaming."""
import pytest
import torch
import torch.nn.functional as F

import encoder_ref as R

pytestmark = pytest.mark.gpu


def make(dtype=torch.float32, right=0, **kw):
    from paper_2607_21271_amd.encoder import EQEncoder
    torch.manual_seed(1)
    args = dict(heads=2, depth=2, sections=(2, 1, 1), left=30, right=right, registers=3)
    args.update(kw)
    return EQEncoder(4, 3, 16, device="cuda", dtype=dtype, **args)


def clip(seed, B=2, N=3, size=16, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(B, N, size, size, 3, 4, generator=g).to(dtype).cuda()


def test_block_against_plain_attention():
    from paper_2607_21271_amd.encoder import EQWindowBlock
    from paper_2607_21271_amd.rotary import grid_positions
    torch.manual_seed(2)
    T, C, H = 4, 32, 4
    block = EQWindowBlock(T, C, H, (2, 1, 1), left=20, right=11, sinks=2, device="cuda")
    pos = grid_positions((2, 5, 5), prefix=2, device="cuda")
    L, D = pos.shape[0], C // H * T
    g = torch.Generator().manual_seed(3)
    x = torch.randn(2, L, C, T, generator=g).cuda()
    with torch.no_grad():
        qkv = block.qkv(block.norm1(x)).view(2, L, 3 * H, D)
        qk = R.rotary(qkv[:, :, :2 * H], pos, block.freqs, (2, 1, 1), T, False)[0].cuda()
        o = _plain(qk[:, :, :H], qk[:, :, H:], qkv[:, :, 2 * H:].double(), L)
        y = x + block.proj(o.float().view(2, L, C, T))
        want = y + block.fc2(F.gelu(block.fc1(block.norm2(y))))
        got = block(x, pos)
    # fp32 sums of some hundred terms through two layers: a few 2^-16 of the largest value
    assert (got - want).abs().max() <= 4 * R.E32 * want.abs().max()


def _plain(q, k, v, L):
    seen = R.visible(L, L, L, 0, 20, 11, 2).cuda()
    s = torch.matmul(q.transpose(1, 2), k.transpose(1, 2).transpose(2, 3).contiguous()) * q.shape[-1] ** -0.5
    a = torch.softmax(s.masked_fill(~seen, float("-inf")), -1)
    return torch.matmul(a, v.transpose(1, 2).contiguous()).transpose(1, 2).contiguous()


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.float16, 2e-2)])
def test_stream_gives_the_whole_clips_tokens(dtype, tol):
    """Tokens frame by frame over caches against the clip at once: the same sums in other orders, and the statistics of
    the same frames; fp16 rounds at every layer of two blocks (2^-11 each, some tens of roundings)."""
    enc = make(dtype)
    x = clip(4, dtype=dtype)
    with torch.no_grad():
        whole, streamed = enc(x), enc.stream(x)
    assert whole.shape == (2, 3 + 3 * 16, 16, 4)
    assert (whole - streamed).abs().max() <= tol * whole.abs().max()
    with pytest.raises(ValueError):
        make(dtype, right=5).stream(x)
    with pytest.raises(ValueError):
        enc(x[:, :, :15])


def test_equivariant_to_the_group():
    """Rotating the frames by 90 degrees and rolling T rolls the tokens' T axis and permutes them in their frame; with
    no positions of rows and columns (time only) the tokens are the same."""
    enc = make(sections=(2, 0, 0), left=-1, right=-1)
    x = clip(5)
    turned = torch.rot90(x, 1, (2, 3)).roll(1, -1)
    with torch.no_grad():
        a, b = enc(x), enc(turned)
    grid = a[:, 3:].view(2, 3, 4, 4, 16, 4)
    err = [((torch.rot90(grid, 1, (2, 3)).roll(s, -1) - b[:, 3:].view_as(grid)).abs().max() / b.abs().max()).item()
           for s in (1, -1)]
    assert min(err) <= 1e-4, err


def test_loss_follows_its_gradient():
    """Every parameter has a gradient, and the loss changes along them at the rate they say (central difference over a
    step that should change the loss by a thousandth; what is left is of third order)."""
    enc = make(right=-1)
    head = torch.nn.Linear(16, 4).cuda()
    params = [*enc.parameters(), *head.parameters()]
    x, y = clip(6, B=4), torch.arange(4).cuda()
    f = lambda: F.cross_entropy(head(enc(x).mean((1, 3))), y)
    loss = f()
    grads = torch.autograd.grad(loss, params)
    assert all(torch.isfinite(g).all() and (g != 0).any() for g in grads)
    square = sum((g.double() ** 2).sum() for g in grads).item()
    step = 1e-3 * loss.item() / square
    ends = []
    with torch.no_grad():
        for s in (1, -2):  # there, and back past the start
            for p, g in zip(params, grads):
                p.add_(g, alpha=s * step)
            ends.append(f().item())
    rate = (ends[0] - ends[1]) / 2 / (step * square)
    assert abs(rate - 1) < 0.02, rate


def test_command_runs(capsys):
    from paper_2607_21271_amd import encoder
    encoder.main(steps=2)
    out = capsys.readouterr().out
    assert "step 1 loss" in out and "streamed against whole clip" in out
