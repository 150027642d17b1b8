"""More rows than a launch of one turn a workgroup may have threads (2^32)."""
import pytest
import torch

import paper_2106_05609_amd as gas

pytestmark = pytest.mark.gpu


def test_rows_of_more_threads_than_a_launch():
    n, f = (1 << 26) + 5, 129                             # 64 threads a row; 35 GB
    x = torch.zeros(n, f, device="cuda")
    rows = torch.tensor([0, 1, n // 2, n - 6, n - 1], device="cuda")
    some = torch.randn(len(rows), f, device="cuda")
    x[rows] = some
    want = torch.empty_like(some)
    gas.gas_residual_norm(some, u=want, pre=gas.NORM_LAYER)
    gas.gas_residual_norm(x, u=x, pre=gas.NORM_LAYER)
    assert torch.equal(x[rows], want) and not x[n - 2].any() and not x[2].any()
    del x
    torch.cuda.empty_cache()
