"""Gates that are nearly open or nearly shut: the gate's gradient goes with g (1 - g), whose smaller factor has float32's digits however small it is, and
the block's share of the stream with g itself."""
import pytest
import torch

import paper_2106_05609_amd as gas
from tests import residual_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def allowed(want, mag, t, f, dtype):
    """As in test_gpu_residual_norm.py, 96 + F / 8 half units of the magnitude; the exponent t log2 e is rounded to half a unit, and its
    factor too, which moves exp(t) by |t| units each."""
    return R.EPS32 * (96 + f / 8 + 4 * t.abs()) * mag + (R.EPS16 * want.abs() if dtype == "bf16" else 0) + 1e-37


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("cols", ["element", "row"])
@pytest.mark.parametrize("n,f", [(70, 1), (65, 3), (90, 8), (40, 16), (33, 64), (130, 47), (20, 256), (9, 600), (7, 1433), (6, 2048), (5, 5000), (3, 9000)])
def test_gates_far_from_the_middle(n, f, cols, dtype):
    gen = torch.Generator().manual_seed(n + f)
    r = lambda *s: torch.randn(*s, generator=gen)
    put = lambda v: v.to(DT[dtype]).cuda()
    a, gh, gu = put(r(n, f)), put(r(n, f)), put(r(n, f))
    t = put((torch.rand(n, f if cols == "element" else 1, generator=gen) - 0.5) * 120)
    p, p_bias, s, q = ((v + 0.3 * r(f)).cuda() for v in (1.0, 0.0, 0.5, 1.0))
    x = torch.zeros_like(a)
    h, stats, gx, ga, gt = torch.empty_like(a), torch.empty(n, 4, device="cuda"), torch.empty_like(a), torch.empty_like(a), torch.empty_like(t)
    gas.gas_residual_norm(x, h=h, a=a, t=t, post=2, p=p, p_bias=p_bias, s=s, alpha=0.7, pre=0, stats=stats)
    d = [v.double().cpu() for v in (a, t, p, p_bias, s, q, gh, gu)]
    A, T, P, PB, S, Q, GH, GU = d
    want, _, st = R.forward(torch.zeros_like(A), A, T, 2, P, PB, S, 0.7, 0, None, None, 1e-5)
    am = (A.abs() + st[:, :1].abs()) * st[:, 1:2]
    mag = 0.7 * S.abs() * torch.sigmoid(T) * ((am + am.amax(1, keepdim=True)) * P.abs() + PB.abs())
    off = (h.double().cpu() - want).abs()
    assert (off <= allowed(want, mag, T, f, dtype)).all(), (off / allowed(want, mag, T, f, dtype)).max()
    # the gradient, beside a stream of ordinary size
    h = put(r(n, f))
    stats[:, 2:] = torch.tensor([0.1, 0.9], device="cuda")
    gas.gas_residual_norm_bwd(gh, gu, h, stats, gx=gx, ga=ga, gt=gt, a=a, t=t, post=2, p=p, p_bias=p_bias, s=s, alpha=0.7, pre=1, q=q)
    _, mag = R.backward(GH, GU, h.double().cpu(), stats.double().cpu(), A, T, T.shape[1], 2, P, PB, S, 0.7, 1, Q)
    want = by_formula(GH, GU, h.double().cpu(), stats.double().cpu(), A, T, P, PB, S, Q)
    off = (gt.double().cpu() - want).abs()
    # mag leaves out the factor 1 - g, which is one of a row or goes with every element
    bound = allowed(want, mag["gt"] * torch.sigmoid(-T), T, f, dtype)
    assert (off <= bound).all(), (off / bound).max()


def by_formula(gh, gu, h, stats, a, t, p, p_bias, s, q):
    """gt with sigmoid(-t) for 1 - g."""
    mean_a, r_a, mean_h, r_h = (c[:, None] for c in stats.unbind(1))
    hn = (h - mean_h) * r_h
    e = gh + r_h * (gu * q - hn * (gu * q * hn).mean(1, keepdim=True))
    each = e * 0.7 * s * ((a - mean_a) * r_a * p + p_bias)
    return (each if t.shape == a.shape else each.sum(1, keepdim=True)) * torch.sigmoid(t) * torch.sigmoid(-t)


@pytest.mark.parametrize("cols", ["element", "row"])
@pytest.mark.parametrize("n,f", [(8000, 1), (4000, 5), (600, 64), (20, 1433), (4, 5000)])
def test_gates_themselves(n, f, cols):
    """h = g and gt = g (1 - g), no norm: |t| up to 80, every step of it some units: the exponential one, its factor's digits and the product's remainder
    one each, 1 + z a half, the reciprocal one, the products a half each: below 16 half units, and 24 for the two factors."""
    gen = torch.Generator().manual_seed(f)
    t = ((torch.rand(n, f if cols == "element" else 1, generator=gen) - 0.5) * 160).cuda()
    a, x = torch.ones(n, f, device="cuda"), torch.zeros(n, f, device="cuda")
    h, gx, gt = torch.empty_like(a), torch.empty_like(a), torch.empty_like(t)
    gas.gas_residual_norm(x, h=h, a=a, t=t)
    gas.gas_residual_norm_bwd(a, None, None, None, gx=gx, gt=gt, a=a, t=t)
    g, rest = torch.sigmoid(t.double()), torch.sigmoid(-t.double())
    off = (h.double() / g - 1).abs().max().item()
    assert off <= 16 * R.EPS32, off / R.EPS32
    off = (gt.double() / (g * rest * (f if cols == "row" else 1)) - 1).abs().max().item()
    # a row's sum: F / 64 additions and six more, whose roundings are half units each
    assert off <= (24 + (f / 64 + 14 if cols == "row" else 0)) * R.EPS32, off / R.EPS32
