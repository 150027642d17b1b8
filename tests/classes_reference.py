"""Losses and top logits of an output layer over many classes in 64 bits from their definitions, with what rounding may move them by.

u = 2^-24, half a unit in the last place of a float32 (2^-8 of a bfloat16). A product's sum over k takes one instruction for 16 terms, each of which
may lose a unit or two of the sum so far and of its own terms: `units(k)` of the sum of the terms' magnitudes."""
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def units(k):
    return 32 + k / 2


def logits(x, w, bias):
    """(z, how far a logit in fp32 may be off): all float64."""
    z, mag = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, mag = z + bias, mag + torch.where(bias.abs() < 1e30, bias.abs(), 0.0)
    return z, U32 * (units(x.shape[1]) * mag + 2 * torch.where(z.abs() < 1e30, z.abs(), 0.0))


def log_sum_exp(z, off):
    """(lse, how far off): the weighted mean of what the logits are off, what the exponents round by, the sums' and the logarithm's."""
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    away = torch.where(p > 0, (z - z.amax(1, keepdim=True)).abs(), 0.0)
    return lse, (p * (off + 4 * U32 * away)).sum(1) + U32 * (120 + z.shape[1] / 256 / 16 + 4 * lse.abs() + 2 * z.amax(1).abs())


def teacher(ids, values, c, t):
    """q and log q [n, k], which entries there are."""
    there = (ids >= 0) & (ids < c) & (values != float("-inf"))
    v = torch.where(there, values.double() / t, float("-inf"))
    some = there.any(1, keepdim=True)
    lse = torch.where(some, torch.logsumexp(torch.where(some, v, 0.0), 1, keepdim=True), 0.0)
    log_q = torch.where(there, v - lse, 0.0)
    return torch.where(there, torch.exp(log_q), 0.0), log_q, there, some[:, 0]


def weights(n, labels, c, some, label_weight):
    """Of the labels' loss and the teacher's."""
    if labels is None:
        return torch.zeros(n, dtype=torch.float64), some.double()
    return label_weight * ((labels >= 0) & (labels < c)).double(), (1 - label_weight) * some.double()


def xent(x, w, bias, labels):
    """{name: (value, how far off)} of loss_rows and lse."""
    z, off = logits(x, w, bias)
    on = (labels >= 0) & (labels < w.shape[1])
    at = torch.where(on, labels, 0).long()[:, None]
    lse, d = log_sum_exp(z, off)
    loss = torch.where(on, lse - z.gather(1, at)[:, 0], 0.0)
    return {"loss": (loss, on * (d + off.gather(1, at)[:, 0] + 2 * U32 * loss.abs())), "lse": (torch.where(on, lse, 0.0), on * d)}


def distill(x, w, bias, ids, values, t, labels, label_weight):
    n, c = x.shape[0], w.shape[1]
    z, off = logits(x, w, bias)
    q, log_q, there, some = teacher(ids, values, c, t)
    a, b = weights(n, labels, c, some, label_weight)
    on = some if labels is None else some | ((labels >= 0) & (labels < c))
    lse, d = log_sum_exp(z, off)
    lse_t, d_t = log_sum_exp(z / t, off / t)
    at = torch.where(there, ids, 0).long()
    zk, ok = z.gather(1, at) / t, off.gather(1, at) / t
    used = q > 0
    kl = torch.where(used, q * (log_q - zk + lse_t[:, None]), 0.0).sum(1)
    k = ids.shape[1]
    # the parts are summed apart: each rounds at its own size; q and its logarithm are of exponents of the teacher's
    far = torch.where(there, values.double().abs() / t, 0.0).amax(1) + 1
    mag = torch.where(used, q * (log_q.abs() + zk.abs()), 0.0).sum(1) + lse_t.abs()
    kl_off = torch.where(used, q * ok, 0.0).sum(1) + d_t + U32 * (k + 16 + 4 * far) * mag
    loss, loss_off = b * t * t * kl, b * t * t * kl_off
    if labels is not None:
        lab = torch.where(a > 0, labels, 0).long()[:, None]
        picked = z.gather(1, lab)[:, 0]
        # a probability of 0 and a weight of 0 are no term
        loss = loss + torch.where(a > 0, a * (lse - picked), 0.0)
        loss_off = loss_off + torch.where(a > 0, a * (d + off.gather(1, lab)[:, 0] + U32 * 8 * (lse.abs() + picked.abs())), 0.0) + U32 * 8 * b * t * t * mag
    pair = torch.stack([lse, lse_t], 1) * on[:, None]
    return {"loss": (torch.where(on, loss, 0.0), on * loss_off), "lse": (pair, torch.stack([d, d_t], 1) * on[:, None])}


def grad_at_logits(x, w, bias, lse, labels, row_scale, ids=None, values=None, t=1.0, label_weight=1.0):
    """(G, how far off in fp32) from lse as given."""
    n, c = x.shape[0], w.shape[1]
    z, off = logits(x, w, bias)
    r = torch.ones(n, dtype=torch.float64) if row_scale is None else row_scale.double()
    g, mag = torch.zeros_like(z), torch.zeros_like(z)

    def softmax(weight, z, off, lse):
        on = (weight != 0)[:, None]
        p = torch.where(on, torch.exp(z - torch.where(on[:, 0], lse, 0.0)[:, None]), 0.0)
        away = torch.where(p > 0, (z - lse[:, None]).abs() + z.abs() + lse.abs()[:, None], 0.0)
        return weight[:, None] * p, weight.abs()[:, None] * p * (off + U32 * (8 + 3 * away))
    if ids is None:
        on = (labels >= 0) & (labels < c)
        a = on.double() * r
        g, mag = softmax(a, z, off, lse.double())
    else:
        q, _, there, some = teacher(ids, values, c, t)
        a, b = weights(n, labels, c, some, label_weight)
        a, b = a * r, b * r
        g1, m1 = softmax(a, z, off, lse[:, 0].double())
        g2, m2 = softmax(b * t, z / t, off / t, lse[:, 1].double())
        g, mag = g1 + g2, m1 + m2
        at, v = torch.where(there, ids, 0).long(), b[:, None] * t * q
        g.scatter_add_(1, at, -v)
        far = torch.where(there, values.double().abs() / t, 0.0).amax(1, keepdim=True) + 1
        mag.scatter_add_(1, at, U32 * v.abs() * (24 + ids.shape[1] / 64 + 4 * far))
    if labels is not None:
        at = torch.where(a != 0, labels, 0).long()[:, None]
        g.scatter_add_(1, at, -a[:, None])
        mag.scatter_add_(1, at, 4 * U32 * a.abs()[:, None])
    return g, mag + 4 * U32 * g.abs()


def gradients(x, w, g, off, scale, bf16, gw_bf16):
    """{name: (value, how far off)} of gx, gw, gbias."""
    s = abs(scale)
    held = off + U16 * g.abs() if bf16 else off + 2 * U32 * g.abs()       # as the products take it
    last = lambda v, rounded: (U16 if rounded else 2 * U32) * v.abs()
    gx, gw, gb = scale * (g @ w.t()), scale * (x.t() @ g), scale * g.sum(0)
    n, c = g.shape
    out = {"gx": (gx, s * (held @ w.abs().t() + U32 * units(c) * (g.abs() @ w.abs().t()))),
           "gw": (gw, s * (x.abs().t() @ held + U32 * units(n) * (x.abs().t() @ g.abs()))),
           "gbias": (gb, s * (off.sum(0) + U32 * units(n) * g.abs().sum(0)))}
    out["gx"] = (gx, out["gx"][1] * (1 + U16) + last(gx, bf16))
    out["gw"] = (gw, out["gw"][1] * (1 + U16) + last(gw, gw_bf16))
    out["gbias"] = (gb, out["gbias"][1] + last(gb, False))
    return out


def top(z, k):
    """(ids, values): the k largest, of equal ones the lower class first, NaN last."""
    key = torch.where(z.isnan(), float("-inf"), z)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    rows = []
    for i in range(z.shape[0]):
        o = order[i]
        nan = z[i][o].isnan()
        rows.append(torch.cat([o[~nan], o[nan].sort().values])[:k])
    ids = torch.stack(rows)
    return ids, z.gather(1, ids)
