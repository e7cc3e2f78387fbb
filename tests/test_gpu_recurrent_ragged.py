"""A ragged batch through the recurrent block and back, against its sequences run alone."""
import pytest
import torch

from test_gpu_recurrent import block

pytestmark = pytest.mark.gpu
LENGTHS = (40, 7, 1, 25)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
def test_gradients_of_a_ragged_batch(kind, post):
    """A loss over the tokens that hold data: gradients of each sequence's tokens and of the gate are those of the sequence
    alone, gradients of padding 0, gradients of parameters the sums over the sequences.

    fp32.  Products of the layers, the scan and the norms are a few dozen sums of up to 256 terms in a row, in an order that may
    differ by the batch; each sum's rounding is under 256 * 2^-24 of its terms, whose absolute values the norms keep within
    ten times of the results: 2^-16 * 10 < 2e-4 of a tensor's largest value."""
    b = block(kind=kind, post_norm=post)
    g = torch.Generator().manual_seed(5)
    x, dy = (torch.randn(len(LENGTHS), 40, 16, 4, generator=g).cuda() for _ in range(2))
    gate = (torch.rand(len(LENGTHS), 16, generator=g) + 0.5).cuda()
    for i, n in enumerate(LENGTHS):
        dy[i, n:] = 0
    params = list(b.parameters())
    grads = lambda x, gate, dy, **kw: torch.autograd.grad(b(x, gate=gate, **kw), [x, gate, *params], dy)
    lengths = torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")
    got = grads(x.requires_grad_(), gate.requires_grad_(), dy, lengths=lengths)
    sums = [torch.zeros_like(p) for p in params]

    def near(a, want, name):
        assert (a - want).abs().max() <= 2e-4 * want.abs().max(), (name, ((a - want).abs().max() / want.abs().max()).item())

    for i, n in enumerate(LENGTHS):
        one = [t.detach().requires_grad_() for t in (x[i:i + 1, :n], gate[i:i + 1])]
        alone = grads(*one, dy[i:i + 1, :n])
        near(got[0][i:i + 1, :n], alone[0], "x %d" % i)
        near(got[1][i:i + 1], alone[1], "gate %d" % i)
        assert (got[0][i, n:] == 0).all()
        for s, a in zip(sums, alone[2:]):
            s += a
    for (name, _), a, s in zip(b.named_parameters(), got[2:], sums):
        near(a, s, name)


def test_padding_that_reaches_the_loss():
    """Gradients of padding through the residual sums and the MLP, which have no lengths: those of the padded tokens alone, whose
    mixer gives out_proj's bias."""
    b = block(post_norm=False)
    g = torch.Generator().manual_seed(6)
    x, dy = (torch.randn(2, 30, 16, 4, generator=g).cuda() for _ in range(2))
    lengths = torch.tensor([30, 12], dtype=torch.int32, device="cuda")
    x.requires_grad_()
    got, = torch.autograd.grad(b(x, lengths=lengths), x, dy)
    pad = x.detach()[1:, 12:].requires_grad_()
    want, = torch.autograd.grad(b(pad, lengths=torch.zeros(1, dtype=torch.int32, device="cuda")), pad, dy[1:, 12:])
    assert (got[1:, 12:] - want).abs().max() <= 2e-4 * want.abs().max()
