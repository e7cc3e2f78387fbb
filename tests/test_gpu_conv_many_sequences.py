"""The causal convolution over more workgroups than a launch takes, on the GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_a_launch_takes():
    """2^20 one-token sequences of 32,776 columns (17 workgroups each, 17.8 million), all of one row read through strides of 0,
    some of them empty: y, 69 GB, holds the row's result where there is a token and 0 elsewhere."""
    from paper_2607_21271_amd.scan import causal_conv
    B, C, T = 1 << 20, 4097, 8
    need = B * C * T * 2
    if torch.cuda.mem_get_info()[0] < 1.5 * need:
        pytest.skip("needs 103 GB of device memory")
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g).half().cuda()
    x, w, b = n(1, 1, C, T), n(C, 4), n(C)
    lengths = (torch.arange(B) % 3 != 1).int().cuda()
    with torch.no_grad():
        want = causal_conv(x, w, b, "silu").view(-1)
        y = causal_conv(x.expand(B, 1, C, T), w, b, "silu", lengths=lengths).view(B, C * T)
        for at in range(0, B, 1 << 14):
            part = y[at:at + (1 << 14)]
            assert torch.equal(part, want * lengths[at:at + (1 << 14), None].half()), at
    del y, part
    torch.cuda.empty_cache()
