"""Rotary positions over more tokens than the workgroups of one launch take."""
import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu


def test_more_tokens_than_one_launch():
    """One token a workgroup (2,049 elements, none of them aligned to more than its own size), 2^24 + 5 tokens turned in
    place: 64 GiB, of which the tokens on either side of a launch's end hold data."""
    from paper_2607_21271_amd import rotary
    L, N, D = (1 << 24) + 5, 3, 683
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB of device memory")
    x = torch.zeros(1, L, N, D, dtype=torch.float16, device="cuda")
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[:, None]
    freqs = rotary.axis_frequencies((2,), device="cuda")
    at = [0, 1, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, L - 1]
    some = torch.randn(1, len(at), N, D, generator=torch.Generator().manual_seed(1)).half().cuda()
    x[:, at] = some
    rotary.rotary_axes_(x, pos, freqs, (2,))
    R.within("y", x[:, at], *R.rotary(some, pos[at], freqs, (2,), 1, False))
    del x
    torch.cuda.empty_cache()
