"""Gradients that leave float32's range, with states of 8 bits and no norm of the gradients to skip the step by."""
import numpy as np
import pytest
import torch

import paper_2106_05609_amd as gas

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan"), 1e25])
@pytest.mark.parametrize("place", [256, 300, 511])
def test_a_block_with_an_infinity_reads_as_nan(bad, place):
    """1e25 is finite and its square is not: v of the block is lost, m is not."""
    n = 1024
    gen = torch.Generator().manual_seed(1)
    g = torch.randn(n, generator=gen).cuda()
    w = torch.randn(n, generator=gen).cuda()
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(n // 256, 2, device="cuda")
    first = g.clone()
    first[place] = bad
    gas.gas_adamw_steps([w], [first], m, v, 1e-3, 1, scales=scales)
    out = [torch.zeros(n, device="cuda") for _ in range(2)]
    gas.gas_adamw_unpack(m, v, scales, *out)
    got_m, got_v = (z.cpu().numpy() for z in out)
    block = np.zeros(n, bool)
    block[256:512] = True
    assert np.isfinite(got_m[~block]).all() and np.isfinite(got_v[~block]).all() and (got_v[~block] > 0).all()
    assert np.isnan(got_v[block]).all()
    assert np.isfinite(got_m[block]).all() if bad == 1e25 else np.isnan(got_m[block]).all()
    # the next step says so in the weights, rather than moving none of them
    gas.gas_adamw_steps([w], [g], m, v, 1e-3, 2, scales=scales)
    w = w.cpu().numpy()
    assert np.isnan(w[block]).all() and np.isfinite(w[~block]).all()


def test_a_block_below_the_normal_numbers_is_nothing():
    """The exception to "a v > 0 is never 0": the block's largest is below the smallest normal number."""
    n = 512
    g = torch.full((n,), 1e-3, device="cuda")
    g[:256] = 1e-19                                       # v = 1e-41
    w, m, v = torch.ones(n, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 2), 7.0, device="cuda")
    gas.gas_adamw_steps([w], [g], m, v, 1e-3, 1, scales=scales)
    assert (v[:256] == 0).all() and scales[0, 1].item() == 0.0 and (v[256:] > 0).all() and scales[1, 1].item() > 0.0
    assert torch.isfinite(w).all()
