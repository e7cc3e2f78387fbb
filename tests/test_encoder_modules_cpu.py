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
