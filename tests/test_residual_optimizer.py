"""What residual.AdamW refuses, without a GPU."""
import pytest
import torch

from paper_2106_05609_amd import residual


def test_bfloat16_tensors_that_share_memory():
    """Each would have a master of its own, and the weights the value of the last one: the others' gradients would be lost."""
    w = torch.zeros(8, 8, dtype=torch.bfloat16)
    other = torch.zeros(8, 8, dtype=torch.bfloat16)
    for tied in ([w, other, w], [w, w[3:]], [other, w[:5], w[4:]]):
        for bits in (8, 32):
            with pytest.raises(ValueError, match="share memory"):
                residual.AdamW(tied, 0.1, bits=bits)
    opt = residual.AdamW([w[:4], w[4:], other, torch.zeros(3), w[:0]], 0.1)
    assert len(opt.tensors) == 5
    f32 = torch.zeros(8)
    residual.AdamW([f32, f32], 0.1)                      # no masters: updated in order
