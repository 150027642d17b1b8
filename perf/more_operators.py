"""The operators of an output layer over many classes, as a list of timed cases: cross-entropy of the layer's logits with its gradients,
distillation from a teacher's top logits with its gradients, and the top logits themselves.  The logits are not an output of any.

`own` chooses between the plain form (elementary torch operations in 32 bits, which hold all logits) and the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOSS, LOSS_BWD, DISTILL, DISTILL_BWD, TOP = "loss", "loss_bwd", "distill", "distill_bwd", "top"
LABEL_WEIGHT = 0.25               # of the labels' loss beside the teacher's


def _case(name, op, rows, width, classes, dtype, bias, labelled=1.0, k=0, temperature=1.0):
    """labelled: the share of the rows that have a label; k: entries of a teacher's row, or of the answer."""
    c = dict(op=op, rows=rows, width=width, classes=classes, dtype=dtype, bias=bias, labelled=labelled, k=k, temperature=temperature)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest batch of a narrow model: latency
        _case("tiny-loss", LOSS, 512, 64, 4_001, "f32", True),
        # a semi-supervised batch of the mid-size community graph: one node in ten has a label
        _case("mid-loss", LOSS, 50_000, 256, 20_000, "f32", False, labelled=0.1),
        # a large vocabulary behind wide rows
        _case("vocabulary-loss", LOSS, 8_192, 2_048, 131_072, "bf16", False),
        # the smallest batch, trained
        _case("tiny-loss-backward", LOSS_BWD, 512, 64, 4_001, "f32", True),
        # odd sizes in everything, some rows without a label
        _case("ragged-loss-backward", LOSS_BWD, 9_973, 300, 50_021, "bf16", True, labelled=0.6),
        # a class for every product of a catalogue, trained
        _case("large-loss-backward", LOSS_BWD, 16_384, 512, 131_072, "bf16", False),
        # a student's loss on a batch of a few thousand rows
        _case("mid-distill", DISTILL, 8_000, 128, 100_003, "bf16", True, k=32, temperature=2.0),
        # a student trained from a teacher and from labels in 32 bits
        _case("mid-distill-backward", DISTILL_BWD, 4_096, 256, 65_536, "f32", False, labelled=0.5, k=64, temperature=2.0),
        # the large batch, trained from a teacher alone
        _case("large-distill-backward", DISTILL_BWD, 16_384, 256, 131_072, "bf16", False, labelled=0.0, k=64, temperature=1.0),
        # one node is asked for
        _case("one-node-top", TOP, 1, 256, 100_003, "bf16", True, k=10),
        # a few requests together, behind wide rows
        _case("few-nodes-top", TOP, 32, 1_024, 250_000, "bf16", False, k=50),
        # a teacher's pass over a batch, its top logits kept for students
        _case("teacher-top", TOP, 8_192, 512, 131_072, "bf16", False, k=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice([LOSS, LOSS_BWD, DISTILL, DISTILL_BWD, TOP])
    dtype, bias = rng.choice(list(DTYPES)), rng.random() < 0.5
    width = rng.choice([64, 128, 256, 512, _log_int(rng, 16, 2_048), _log_int(rng, 16, 2_048)])
    classes = rng.choice([_log_int(rng, 500, 262_144), _log_int(rng, 2_000, 262_144), 8 * _log_int(rng, 250, 32_768)])
    most = min(50_000, 1_000_000_000 // classes, 400_000_000_000 // (classes * width))
    rows = _log_int(rng, 1, max(2, most))
    if op in (LOSS, LOSS_BWD):
        return _case(None, op, rows, width, classes, dtype, bias, labelled=rng.choice([1.0, round(rng.uniform(0.05, 1.0), 2)]))
    if op == TOP:
        return _case(None, op, rows, width, classes, dtype, bias, k=_log_int(rng, 1, 128))
    return _case(None, op, rows, width, classes, dtype, bias, labelled=rng.choice([0.0, 1.0, round(rng.uniform(0.05, 1.0), 2)]),
                 k=_log_int(rng, 1, 128), temperature=rng.choice([1.0, 2.0, round(rng.uniform(0.5, 5.0), 1)]))


def _normal(gen, shape, scale=1.0):
    return torch.empty(shape, device="cuda").normal_(generator=gen).mul_(scale)


def _labelled(case):
    """How many rows have a label."""
    return min(case["rows"], math.ceil(case["labelled"] * case["rows"]))


def _statistics(s):
    """What the forward call leaves for the backward one: the logarithm of the sum of exponentials, at every temperature that it needs."""
    z = s["x"].float() @ s["w"].float()
    if s["bias"] is not None:
        z += s["bias"].float()
    if s["case"]["op"] == LOSS_BWD:
        return torch.logsumexp(z, 1)
    return torch.stack([torch.logsumexp(z, 1), torch.logsumexp(z.div_(s["case"]["temperature"]), 1)], 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, f, c, k, dt, op = case["rows"], case["width"], case["classes"], case["k"], DTYPES[case["dtype"]], case["op"]
    s = dict(case=case)
    # rows of a norm and a layer that leaves logits of about one; where classes are put in order, both in steps as quantised values
    # have them, so that their products are whole in 32 bits in any order and equal logits are equal
    grid = (lambda t, step: t.div_(step).round_().mul_(step)) if op == TOP else (lambda t, step: t)
    s["x"] = grid(_normal(gen, (n, f)), 1 / 16).to(dt)
    s["w"] = grid(_normal(gen, (f, c), 1.5 / math.sqrt(f)), 1 / 512).to(dt)
    s["bias"] = grid(_normal(gen, (c,), 0.3), 1 / 512).to(dt) if case["bias"] else None
    if op == TOP:
        s["ids"], s["values"] = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
        s["lse"] = torch.empty(n, device="cuda")
        return s
    # a few classes have most of the labels
    labels = torch.rand(n, generator=gen, device="cuda").pow_(3).mul_(c).to(torch.int32).clamp_(max=c - 1)
    labels[torch.randperm(n, generator=gen, device="cuda")[_labelled(case):]] = -1
    s["labels"] = labels if op in (LOSS, LOSS_BWD) or case["labelled"] > 0 else None
    if op in (DISTILL, DISTILL_BWD):
        # distinct classes in no order; a teacher's logits fall off from the first on; some rows have fewer entries
        gaps = torch.randint(1, max(2, c // k), (n, k), generator=gen, device="cuda")
        start = torch.randint(0, c, (n, 1), generator=gen, device="cuda")
        order = torch.rand(n, k, generator=gen, device="cuda").argsort(1)
        ids = ((start + gaps.cumsum(1)) % c).gather(1, order)
        fewer = torch.rand(n, 1, generator=gen, device="cuda") < 0.1
        held = torch.where(fewer, torch.randint(0, k + 1, (n, 1), generator=gen, device="cuda"), k)
        s["ids"] = torch.where(torch.arange(k, device="cuda") < held, ids, -1).to(torch.int32)
        s["values"] = 6.0 - torch.empty(n, k, device="cuda").exponential_(4.0, generator=gen).cumsum(1)
    if op in (LOSS, DISTILL):
        s["loss"], s["sum"] = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
        s["lse"] = torch.empty((n,) if op == LOSS else (n, 2), device="cuda")
        return s
    s["lse"] = _statistics(s)
    s["scale"] = 1.0 / max(1, _labelled(case) if op == LOSS_BWD else n)
    s["gx"], s["gw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    s["gbias"] = torch.empty(c, device="cuda") if case["bias"] else None
    return s


# ---- the plain forms

def _logits(s):
    z = s["x"].float() @ s["w"].float()
    return z if s["bias"] is None else z + s["bias"].float()


def _log_sum_exp(z):
    most = z.amax(1, keepdim=True)
    return (most + torch.log(torch.exp(z - most).sum(1, keepdim=True)))[:, 0]


def _teacher(s):
    """The teacher's distribution over the entries of a row, its logarithm, the classes (0 for an entry that is not there), which rows have any."""
    there = s["ids"] >= 0
    t = torch.where(there, s["values"] / s["case"]["temperature"], float("-inf"))
    some = there.any(1)
    most = torch.where(some[:, None], t.amax(1, keepdim=True), 0.0)
    e = torch.exp(t - most)
    total = torch.where(some[:, None], e.sum(1, keepdim=True), 1.0)
    return e / total, torch.where(there, t - most, 0.0) - torch.log(total), s["ids"].long().clamp(min=0), some


def _weights(s):
    """Of the labels' loss and of the teacher's in every row."""
    n, dev = s["case"]["rows"], s["x"].device
    if s["labels"] is None:
        return torch.zeros(n, device=dev), torch.ones(n, device=dev)
    return (s["labels"] >= 0).float() * LABEL_WEIGHT, torch.full((n,), 1 - LABEL_WEIGHT, device=dev)


def _plain_loss(s):
    z, labelled = _logits(s), s["labels"] >= 0
    lse = _log_sum_exp(z)
    loss = lse - z.gather(1, s["labels"].long().clamp(min=0)[:, None])[:, 0]
    loss, lse = torch.where(labelled, loss, 0.0), torch.where(labelled, lse, 0.0)
    return {"loss": loss, "lse": lse, "sum": loss.double().sum().float().reshape(1)}


def _gradients(s, g):
    """From the gradient at the logits."""
    dt, scale = s["x"].dtype, s["scale"]
    out = {"gx": (g @ s["w"].float().t()).mul_(scale).to(dt), "gw": (s["x"].float().t() @ g).mul_(scale).to(dt)}
    if s["gbias"] is not None:
        out["gbias"] = g.sum(0) * scale
    return out


def _plain_loss_bwd(s):
    labelled = (s["labels"] >= 0).float()[:, None]
    g = torch.exp(_logits(s) - s["lse"][:, None]).mul_(labelled)
    g.scatter_add_(1, s["labels"].long().clamp(min=0)[:, None], -labelled)
    return _gradients(s, g)


def _plain_distill(s):
    z, t = _logits(s), s["case"]["temperature"]
    q, log_q, ids, some = _teacher(s)
    label_weight, weight = _weights(s)
    lse, lse_t = _log_sum_exp(z), _log_sum_exp(z / t)
    loss = torch.where(some, weight * t * t * (q * (log_q - z.gather(1, ids) / t + lse_t[:, None])).sum(1), 0.0)
    counted = some
    if s["labels"] is not None:
        labelled = s["labels"] >= 0
        picked = z.gather(1, s["labels"].long().clamp(min=0)[:, None])[:, 0]
        loss = loss + label_weight * (lse - picked)
        counted = some | labelled
    lse = torch.where(counted[:, None], torch.stack([lse, lse_t], 1), 0.0)
    return {"loss": loss, "lse": lse, "sum": loss.double().sum().float().reshape(1)}


def _plain_distill_bwd(s):
    z, t = _logits(s), s["case"]["temperature"]
    q, _, ids, some = _teacher(s)
    label_weight, weight = _weights(s)
    weight = (weight * t * some)[:, None]
    g = torch.exp(z / t - s["lse"][:, 1:]).mul_(weight)
    g.scatter_add_(1, ids, -weight * q)
    if s["labels"] is not None:
        g += torch.exp(z - s["lse"][:, :1]).mul_(label_weight[:, None])
        g.scatter_add_(1, s["labels"].long().clamp(min=0)[:, None], -label_weight[:, None])
    return _gradients(s, g)


def _plain_top(s):
    z, k = _logits(s), s["case"]["k"]
    lse = _log_sum_exp(z)
    # a whole number for every logit, larger for larger ones and, of equal ones, for those of lower classes
    z = z + 0.0
    bits = z.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
    key += torch.arange(z.shape[1] - 1, -1, -1, device=z.device)
    ids = z.shape[1] - 1 - (torch.topk(key, k, 1).values & 0xFFFFFFFF)
    return {"ids": ids.to(torch.int32), "values": z.gather(1, ids), "lse": lse}


PLAIN = {LOSS: _plain_loss, LOSS_BWD: _plain_loss_bwd, DISTILL: _plain_distill, DISTILL_BWD: _plain_distill_bwd, TOP: _plain_top}


def run(s):
    op = s["case"]["op"]
    if not own:
        return PLAIN[op](s)
    import paper_2106_05609_amd as gas
    x, w, bias = s["x"], s["w"], s["bias"]
    if op == TOP:
        gas.gas_linear_top(x, w, s["ids"], s["values"], lse=s["lse"], bias=bias)
        return {"ids": s["ids"], "values": s["values"], "lse": s["lse"]}
    if op == LOSS:
        gas.gas_linear_xent(x, w, s["labels"], s["loss"], s["lse"], bias=bias, loss_sum=s["sum"])
    elif op == LOSS_BWD:
        gas.gas_linear_xent_bwd(x, w, s["labels"], s["lse"], gx=s["gx"], gw=s["gw"], gbias=s["gbias"], bias=bias, scale=s["scale"])
    else:
        same = dict(bias=bias, labels=s["labels"], label_weight=LABEL_WEIGHT, temperature=s["case"]["temperature"])
        if op == DISTILL:
            gas.gas_linear_distill(x, w, s["ids"], s["values"], s["loss"], s["lse"], loss_sum=s["sum"], **same)
        else:
            gas.gas_linear_distill_bwd(x, w, s["ids"], s["values"], s["lse"], gx=s["gx"], gw=s["gw"], gbias=s["gbias"], scale=s["scale"], **same)
    if op in (LOSS, DISTILL):
        return {"loss": s["loss"], "lse": s["lse"], "sum": s["sum"]}
    return {name: s[name] for name in ("gx", "gw", "gbias") if s[name] is not None}


def work(case):
    n, f, c, k, eb = case["rows"], case["width"], case["classes"], case["k"], 4 if case["dtype"] == "f32" else 2
    counted = _labelled(case) if case["op"] in (LOSS, LOSS_BWD) else n       # rows without a label have no product
    read = eb * (counted * f + f * c + (c if case["bias"] else 0))
    if case["op"] == TOP:
        return dict(bytes=read + n * (8 * k + 4), flops=2 * n * f * c)
    targets = 4 * n if case["op"] in (LOSS, LOSS_BWD) else 8 * n * k + (4 * n if case["labelled"] > 0 else 0)
    statistics = 4 * n if case["op"] in (LOSS, LOSS_BWD) else 8 * n
    if case["op"] in (LOSS, DISTILL):
        return dict(bytes=read + targets + statistics + 4 * n, flops=2 * counted * f * c)
    written = eb * (n * f + f * c) + (4 * c if case["bias"] else 0)
    return dict(bytes=read + targets + statistics + written, flops=6 * counted * f * c)


# ---- the definitions in 64 bits

def _exact_logits(s):
    z = torch.mm(s["x"].double(), s["w"].double())
    if s["bias"] is not None:
        z.add_(s["bias"].double()[None, :])
    return z


def _one_hot_minus(g, rows, columns, values):
    """g[rows, columns] -= values, entry by entry of a row in turn."""
    flat = g.view(-1)
    flat.index_add_(0, rows * g.shape[1] + columns, values, alpha=-1.0)
    return g


def _exact_teacher(s):
    """For every entry that is there: its row, class, and the logarithm of its probability."""
    rows, places = torch.nonzero(s["ids"] >= 0, as_tuple=True)
    columns, t = s["ids"][rows, places].long(), s["values"][rows, places].double() / s["case"]["temperature"]
    n = s["case"]["rows"]
    most = torch.full((n,), -math.inf, dtype=torch.float64, device=t.device).scatter_reduce(0, rows, t, "amax")
    total = torch.zeros(n, dtype=torch.float64, device=t.device).index_add_(0, rows, (t - most[rows]).exp())
    return rows, columns, t - most[rows] - total.log()[rows]


def _exact_forward(s):
    z, case = _exact_logits(s), s["case"]
    n, dev = case["rows"], z.device
    loss, counted = torch.zeros(n, dtype=torch.float64, device=dev), torch.zeros(n, dtype=torch.bool, device=dev)
    lse = torch.logsumexp(z, 1)
    share = 1.0 if case["op"] == LOSS else LABEL_WEIGHT
    if s["labels"] is not None:
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        loss[rows] += share * (lse[rows] - z[rows, s["labels"][rows].long()])
        counted[rows] = True
    if case["op"] == DISTILL:
        t = case["temperature"]
        rows, columns, log_q = _exact_teacher(s)
        picked = z[rows, columns] / t
        lse_t = torch.logsumexp(z.div_(t), 1)
        kl = log_q.exp() * (log_q - picked + lse_t[rows])
        loss.index_add_(0, rows, kl, alpha=t * t * (1.0 if s["labels"] is None else 1.0 - share))
        counted[rows] = True
        lse = torch.stack([lse, lse_t], 1) * counted[:, None]
    else:
        lse = lse * counted
    return {"loss": loss, "lse": lse, "sum": loss.sum().reshape(1)}


def _exact_backward(s):
    z, case, lse = _exact_logits(s), s["case"], s["lse"].double()
    labels = s["labels"]
    share = 1.0 if case["op"] == LOSS_BWD else LABEL_WEIGHT
    if case["op"] == DISTILL_BWD:
        t = case["temperature"]
        rows, columns, log_q = _exact_teacher(s)
        weight = torch.zeros(case["rows"], dtype=torch.float64, device=z.device)
        weight[rows] = t * (1.0 if labels is None else 1.0 - share)
        g = (z / t).sub_(lse[:, 1:2]).exp_().mul_(weight[:, None])
        _one_hot_minus(g, rows, columns, log_q.exp() * weight[rows])
    else:
        g = torch.zeros_like(z)
    if labels is not None:
        rows = torch.nonzero(labels >= 0)[:, 0]
        one = lse[:, :1] if lse.dim() == 2 else lse[:, None]
        g[rows] += z[rows].sub_(one[rows]).exp_().mul_(share)
        _one_hot_minus(g, rows, labels[rows].long(), torch.full_like(rows, 1, dtype=torch.float64) * share)
    del z
    g.mul_(s["scale"])
    out = {"gx": torch.mm(s["w"].double(), g.t()).t().contiguous(), "gw": torch.mm(g.t(), s["x"].double()).t().contiguous()}
    if s["gbias"] is not None:
        out["gbias"] = torch.mv(g.t(), torch.ones(g.shape[0], dtype=torch.float64, device=g.device))
    return out


def _exact_top(s):
    ids, values, lse = [], [], []
    for first in range(0, s["case"]["rows"], 1024):
        z = _exact_logits(dict(s, x=s["x"][first:first + 1024]))
        lse.append(torch.logsumexp(z, 1))
        best = torch.sort(z, dim=1, descending=True, stable=True)
        ids.append(best.indices[:, :s["case"]["k"]].to(torch.int32))
        values.append(best.values[:, :s["case"]["k"]].clone())
    return {"ids": torch.cat(ids), "values": torch.cat(values), "lse": torch.cat(lse)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == TOP:
        return _exact_top(s)
    return (_exact_forward if case["op"] in (LOSS, DISTILL) else _exact_backward)(s)
