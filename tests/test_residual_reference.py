"""The 64-bit definitions of the norms with gate and residual scale against themselves: gradients by the formulas, by automatic
differentiation and by differences."""
import itertools

import pytest
import torch

from tests import residual_reference as R


def _case(n, f, kind, gate, bias, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    vec = lambda around: around + 0.3 * r(f)
    return dict(x=r(n, f), a=r(n, f), t=None if gate == 0 else r(n, gate), post=kind, p=vec(1.0), p_bias=vec(0.0) if bias else None, s=vec(0.5),
                alpha=0.7, pre=kind, q=vec(1.0), q_bias=vec(0.0) if bias else None, eps=1e-3)


@pytest.mark.parametrize("kind,gate,bias", itertools.product((R.NONE, R.RMS, R.LAYER), (0, 1, 6), (False, True)))
def test_gradients(kind, gate, bias):
    c = _case(5, 6, kind, gate, bias)
    leaves = {k: v.requires_grad_() for k, v in c.items() if torch.is_tensor(v)}
    gh, gu = torch.randn(5, 6, dtype=torch.float64), torch.randn(5, 6, dtype=torch.float64)

    def loss(**kw):
        h, u, _ = R.forward(**{**c, **kw})
        return (h * gh).sum() + (u * gu).sum()
    loss().backward()
    h, _, stats = R.forward(**c)
    got, mag = R.backward(gh, gu, h.detach(), stats.detach(), *(None if c[k] is None else c[k].detach() for k in ("a", "t")), gate, kind,
                          *(None if c[k] is None else c[k].detach() for k in ("p", "p_bias", "s")), 0.7, kind, c["q"].detach())
    for k, leaf in leaves.items():
        assert torch.allclose(got["g" + k], leaf.grad, rtol=1e-11, atol=1e-12), k
        assert (mag["g" + k] >= got["g" + k].abs() * (1 - 1e-9)).all()
        direction = torch.randn_like(leaf)
        with torch.no_grad():
            step = 1e-5
            slope = (loss(**{k: leaf + step * direction}) - loss(**{k: leaf - step * direction})) / (2 * step)
        assert abs(slope - (leaf.grad * direction).sum()) <= 1e-7 * (1 + leaf.grad.norm() * direction.norm()), k


def test_workspace_of_the_backward_pass_serves_fewer_rows():
    from paper_2106_05609_amd import binding as B
    for f in (1, 7, 47, 64, 100, 256, 520, 1433, 2000, 5000, 9000):
        last = 0
        for n in [*range(0, 3000, 7), 21_248, 50_000, 50_001, 262_143, 600_000, 3_125_002]:
            need = B.gas_residual_norm_bwd_workspace(n, f)
            assert need >= last, (n, f)
            last = need
