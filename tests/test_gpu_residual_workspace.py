"""The backward call of the norms takes a workspace of what its type needs, and refuses a smaller one."""
import pytest
import torch

import paper_2106_05609_amd as gas

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,f", [(1, 8), (5000, 256), (70_001, 600), (140_000, 64), (300, 5000), (100, 9000)])
def test_as_much_as_the_type_needs(n, f, dtype):
    need = gas.gas_residual_norm_bwd_workspace(n, f, dtype)
    assert 0 < need <= gas.gas_residual_norm_bwd_workspace(n, f)
    gh, h = (torch.randn(n, f, device="cuda").to(dtype) for _ in range(2))
    stats = torch.tensor([[0.0, 1.0, 0.1, 0.9]], device="cuda").repeat(n, 1)
    gq, gx = torch.zeros(f, device="cuda"), torch.empty_like(gh)
    room = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
    call = lambda size: gas.gas_residual_norm_bwd(None, gh, h, stats, gx=gx, pre=2, gq=gq, workspace=room[:size])
    call(need)
    assert (room[need:] == 77).all()
    hn = (h.double() - stats[:, 2:3].double()) * stats[:, 3:].double()
    want, mag = (gh.double() * hn).sum(0), (gh.double() * hn).abs().sum(0)
    assert ((gq.double() - want).abs() <= (96 + f / 8 + 64 + n / 16) * 2.0 ** -24 * mag).all()
    with pytest.raises(gas.GasError, match=f"{need - 16} bytes, {need} are needed"):
        call(need - 16)
