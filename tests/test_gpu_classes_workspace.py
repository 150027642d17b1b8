"""Calls of an output layer over many classes write nothing beyond the workspace that they ask for, whatever their sizes choose and however many rows count."""
import pytest
import torch

import paper_2106_05609_amd as gas
from tests.test_gpu_classes import DT, exact_layer, with_teacher

pytestmark = pytest.mark.gpu
SIZES = [(1, 64, 500), (3, 1100, 700), (8, 256, 29_360), (8, 40, 5001), (9, 1030, 600), (40, 200, 9000), (64, 2048, 264), (65, 33, 511), (100, 2048, 1500),
         (200, 5000, 520), (300, 1433, 264), (520, 70, 40_000), (30, 8200, 300), (40, 600, 33_001)]


def room(need):
    """`need` bytes and the 64 KB behind them, all ones."""
    whole = torch.full((need + 65536,), 255, dtype=torch.uint8, device="cuda")
    return whole[:need], whole[need:]


@pytest.mark.parametrize("n, f, c", SIZES)
@pytest.mark.parametrize("dtype", list(DT))
def test_nothing_beyond_it(n, f, c, dtype):
    dt, k = DT[dtype], 5
    new = lambda *shape: torch.empty(shape, device="cuda")
    for labelled in (1.0, 0.4, 0.0):
        s, _ = with_teacher(n, f, c, k, dtype, labelled)
        grads = lambda: dict(gx=torch.empty_like(s["x"]), gw=new(f, c), gbias=new(c))
        calls = [(gas.gas_linear_xent_workspace(n, f, c, dt), gas.gas_linear_xent, (s["labels"], new(n), new(n)), dict(bias=s["bias"])),
                 (gas.gas_linear_xent_bwd_workspace(n, f, c, dt), gas.gas_linear_xent_bwd, (s["labels"], torch.full((n,), 9.0, device="cuda")), grads()),
                 (gas.gas_linear_distill_workspace(n, f, c, dt, k), gas.gas_linear_distill, (s["ids"], s["values"], new(n), new(n, 2)), dict(labels=s["labels"], temperature=1.5)),
                 (gas.gas_linear_distill_bwd_workspace(n, f, c, dt, k), gas.gas_linear_distill_bwd, (s["ids"], s["values"], torch.full((n, 2), 9.0, device="cuda")),
                  dict(grads(), temperature=2.0))]
        for need, call, args, kw in calls:
            work, beyond = room(need)
            call(s["x"], s["w"], *args, workspace=work, **kw)
            assert (beyond == 255).all(), (call.__name__, labelled)
    s = exact_layer(n, f, c, dtype)
    work, beyond = room(gas.gas_linear_top_workspace(n, f, c, dt, 33))
    gas.gas_linear_top(s["x"], s["w"], torch.empty(n, 33, dtype=torch.int32, device="cuda"), new(n, 33), lse=new(n), bias=s["bias"], workspace=work)
    assert (beyond == 255).all()
