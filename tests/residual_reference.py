"""The norms before and after a block with gate and residual scale, and AdamW, in 64 bits from their definitions, with the magnitude of
what every result is summed from: rounding errors are relative to that."""
import numpy as np
import torch

NONE, RMS, LAYER = 0, 1, 2
EPS32, EPS16 = 2.0 ** -24, 2.0 ** -8      # half a unit in the last place of 1: float32 has 24 bits, bfloat16 8


def _stats(z, kind, eps):
    mean = z.mean(1, keepdim=True) if kind == LAYER else z.new_zeros(z.shape[0], 1)
    r = z.new_ones(z.shape[0], 1) if kind == NONE else 1 / ((z - mean).square().mean(1, keepdim=True) + eps).sqrt()
    return mean, r


def forward(x, a, t, post, p, p_bias, s, alpha, pre, q, q_bias, eps):
    """(h, u, stats), all arguments float64 tensors or None."""
    one, zero = x.new_ones(x.shape[1]), x.new_zeros(x.shape[1])
    or_ = lambda v, otherwise: otherwise if v is None else v
    h, mean_a, r_a = x, x.new_zeros(x.shape[0], 1), x.new_ones(x.shape[0], 1)
    if a is not None:
        mean_a, r_a = _stats(a, post, eps)
        y = (a - mean_a) * r_a * or_(p, one) + or_(p_bias, zero)
        g = 1.0 if t is None else torch.sigmoid(t)
        h = x + alpha * or_(s, one) * g * y
    mean_h, r_h = _stats(h, pre, eps)
    u = (h - mean_h) * r_h * or_(q, one) + or_(q_bias, zero)
    return h, u, torch.cat([mean_a, r_a, mean_h, r_h], 1)


def backward(gh, gu, h, stats, a, t, gate_cols, post, p, p_bias, s, alpha, pre, q):
    """({name: gradient}, {name: magnitude}) by the formulas, h and stats as given."""
    like = next(v for v in (gh, gu) if v is not None)
    n, f = like.shape
    one, zero = like.new_ones(f), like.new_zeros(f)
    or_ = lambda v, otherwise: otherwise if v is None else v
    stats = like.new_tensor([[0.0, 1.0, 0.0, 1.0]]).expand(n, 4) if stats is None else stats
    mean_a, r_a, mean_h, r_h = (c[:, None] for c in stats.unbind(1))
    mean = lambda z: z.sum(1, keepdim=True) / f
    out, mag = {}, {}

    def jacobian(d, z, r, kind, dm, zm):
        along = torch.zeros_like(r) if kind == NONE else mean(d * z)
        flat = mean(d) if kind == LAYER else torch.zeros_like(r)
        return r * (d - flat - z * along), r * (dm + (mean(dm) if kind == LAYER else 0) + (zm * mean(dm * zm) if kind != NONE else 0))
    gh, e_mag = or_(gh, torch.zeros_like(like)), or_(gh, torch.zeros_like(like)).abs()
    e = gh
    if gu is not None:
        hn, hm = (h - mean_h) * r_h, (h.abs() + mean_h.abs()) * r_h
        more, m = jacobian(gu * or_(q, one), hn, r_h, pre, (gu * or_(q, one)).abs(), hm)
        e, e_mag = gh + more, e_mag + m
        out["gq"], mag["gq"] = (gu * hn).sum(0), (gu.abs() * hm).sum(0)
        out["gq_bias"], mag["gq_bias"] = gu.sum(0), gu.abs().sum(0)
    out["gx"], mag["gx"] = e, e_mag
    if a is None:
        return out, mag
    an, am = (a - mean_a) * r_a, (a.abs() + mean_a.abs()) * r_a
    y, ym = an * or_(p, one) + or_(p_bias, zero), am * or_(p, one).abs() + or_(p_bias, zero).abs()
    g = torch.ones_like(a) if t is None else torch.sigmoid(t).expand(n, f)
    k = alpha * or_(s, one) * g
    dy, dym = e * k, e_mag * k.abs()
    out["gs"], mag["gs"] = (e * alpha * g * y).sum(0), (e_mag * abs(alpha) * g * ym).sum(0)
    out["gp"], mag["gp"] = (dy * an).sum(0), (dym * am).sum(0)
    out["gp_bias"], mag["gp_bias"] = dy.sum(0), dym.sum(0)
    if t is not None:
        gt, gtm = dy * y * (1 - g), dym * ym * 1.0
        if gate_cols == 1:
            gt, gtm = gt.sum(1, keepdim=True), gtm.sum(1, keepdim=True)
        out["gt"], mag["gt"] = gt, gtm
    c = dy * or_(p, one)
    out["ga"], mag["ga"] = jacobian(c, an, r_a, post, dym * or_(p, one).abs(), am)
    return out, mag


# ---- AdamW
def layout(sizes):
    """First element of every tensor in the state, and the state's elements."""
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // 256) * 256
    return starts, at


def decode(m, v, scales):
    k = m.astype(np.float64).reshape(-1, 256)
    j = v.astype(np.float64).reshape(-1, 256)
    scales = scales.astype(np.float64).reshape(-1, 2)
    return (scales[:, :1] * k * np.abs(k) / 127.0 ** 2).reshape(-1), (scales[:, 1:] * (j / 255.0) ** 4).reshape(-1)


def adamw(w, g, m, v, lr, t, b1, b2, eps, wd, c=1.0):
    """(w, m, v) after a step, float64 arrays of one tensor."""
    g = g * c
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return w - lr * wd * w - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v
