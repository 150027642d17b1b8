"""The operators of deep residual models and their training, as a list of timed cases: the norms before and after a block with its
gate and residual scale (forward, backward), the squared norm of a model's gradients, and AdamW over all of its tensors with
states in 32 bits or in 8.

`own` chooses between the plain form (elementary torch operations in 32 bits) and the framework's calls.
"""
import math

import torch

own = False

EPS = 1e-5                        # of the norms
LR, BETA1, BETA2, ADAM_EPS, STEP = 3e-4, 0.9, 0.999, 1e-8, 17
BLOCK = 256                       # elements that share a scale; tensors start at multiples of it
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KINDS = {"none": 0, "rms": 1, "layer": 2}
FORWARD, BACKWARD, NORM, ADAMW = "forward", "backward", "sq_norms", "adamw"


def _rows(name, op, rows, width, dtype, norm, gate, bias, push=False):
    c = dict(op=op, rows=rows, width=width, dtype=dtype, norm=norm, gate=gate, bias=bias, push=push)
    return dict(c, name=name) if name else c


def _params(name, op, f_in, hidden, f_out, layers, table=0, dtype="f32", bits=32, master=False):
    c = dict(op=op, f_in=f_in, hidden=hidden, f_out=f_out, layers=layers, table=table, dtype=dtype, bits=bits, master=master)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one node is asked for: a layer's norms over a single row, nothing but latency
        _rows("one-node-forward", FORWARD, 1, 256, "bf16", "rms", "full", False),
        # one batch of the mid-size community graph, its normed rows pushed to the next layer's history table
        _rows("mid-forward-push", FORWARD, 50_000, 256, "f32", "layer", "full", True, push=True),
        # one batch of the huge power-law graph in bf16: inference at the largest size
        _rows("huge-forward", FORWARD, 3_125_002, 256, "bf16", "rms", "full", False),
        # a citation-sized batch of a narrow model, trained
        _rows("tiny-backward", BACKWARD, 512, 64, "f32", "layer", "full", True),
        # bag-of-words features normed as they come: a width that nothing divides, one gate per node
        _rows("ragged-backward", BACKWARD, 19_997, 1433, "bf16", "layer", "row", True),
        # one batch of the large power-law graph, trained
        _rows("large-backward", BACKWARD, 600_000, 256, "f32", "rms", "full", False),
        # clipping: the gradients of the deep narrow model, many small matrices; and of a learned embedding of every node
        _params("deep-norm", NORM, 128, 64, 64, 64),
        _params("table-norm", NORM, 128, 64, 47, 3, table=2_400_000),
        # the step of a two-layer model: launches and host time
        _params("tiny-adamw", ADAMW, 64, 64, 64, 1),
        # the step of the deep narrow model, 32 bits and 8
        _params("deep-adamw8", ADAMW, 128, 64, 64, 64, bits=8),
        # a stack of wide layers
        _params("wide-adamw", ADAMW, 1433, 2048, 47, 16),
        # a learned embedding of every node, bf16 weights beside their 32-bit masters, states in 8 bits
        _params("table-adamw8", ADAMW, 128, 64, 47, 3, table=2_400_000, dtype="bf16", bits=8, master=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice([FORWARD, BACKWARD, FORWARD, BACKWARD, NORM, ADAMW, ADAMW])
    if op in (FORWARD, BACKWARD):
        width = rng.choice([64, 100, 128, 256, 512, _log_int(rng, 8, 2048), _log_int(rng, 8, 2048)])
        dtype = rng.choice(list(DTYPES))
        most = min(3_000_000, 150_000_000 // width)
        return _rows(None, op, _log_int(rng, 1, most), width, dtype, rng.choice(["rms", "layer"]),
                     rng.choice(["none", "full", "full", "row"]), rng.random() < 0.5, op == FORWARD and rng.random() < 0.4)
    hidden = _log_int(rng, 16, 512)
    table = rng.choice([0, 0, _log_int(rng, 1000, 100_000_000 // hidden)])
    dtype = rng.choice(list(DTYPES)) if op == ADAMW else "f32"
    return _params(None, op, _log_int(rng, 16, 1433), hidden, rng.randint(2, 64), rng.randint(1, 80), table, dtype,
                   rng.choice([8, 32]) if op == ADAMW else 32, dtype == "bf16" and rng.random() < 0.7)


def _sizes(case):
    """Elements of every tensor of a model: input and output products, a product and two gains for each layer, an embedding."""
    h = case["hidden"]
    sizes = [case["f_in"] * h, h * case["f_out"]] + case["layers"] * [h * h, h, h]
    return sizes + ([case["table"] * h] if case["table"] else [])


def _decays(case):
    """Weight decay of every tensor: gains have none."""
    return [0.01, 0.01] + case["layers"] * [0.01, 0.0, 0.0] + ([0.01] if case["table"] else [])


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _normal(gen, shape, scale=1.0, dtype=torch.float32):
    out = torch.empty(shape, device="cuda", dtype=torch.float32).normal_(generator=gen)
    return out.mul_(scale).to(dtype)


def _norm_stats(z, kind, eps):
    mean = z.mean(1) if kind == "layer" else z.new_zeros(z.shape[0])
    return mean, torch.rsqrt((z - mean[:, None]).square().mean(1) + eps)


def _prepare_rows(case, gen):
    n, f, dt, kind = case["rows"], case["width"], DTYPES[case["dtype"]], case["norm"]
    s = dict(case=case, alpha=0.5)
    s["a"] = _normal(gen, (n, f), 0.7, dt)
    s["t"] = None if case["gate"] == "none" else _normal(gen, (n, f if case["gate"] == "full" else 1), 1.0, dt)
    vector = lambda around, spread: _normal(gen, (f,), spread).add_(around)
    s["p"], s["s"], s["q"] = vector(1.0, 0.1), vector(0.5, 0.1), vector(1.0, 0.1)
    s["p_bias"], s["q_bias"] = (vector(0.0, 0.1), vector(0.0, 0.1)) if case["bias"] else (None, None)
    empty = lambda like: None if like is None else torch.empty_like(like)
    if case["op"] == FORWARD:
        s["x"] = _normal(gen, (n, f), 1.5, dt)
        s["h"], s["u"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["idx"] = s["hist"] = None
        if case["push"]:
            s["idx"] = torch.randperm(4 * n, generator=gen, device="cuda")[:n].to(torch.int32)
            s["hist"] = torch.zeros(4 * n, f, dtype=dt, device="cuda")
        return s
    s["gh"], s["gu"] = _normal(gen, (n, f), 0.1, dt), _normal(gen, (n, f), 0.1, dt)
    h = _normal(gen, (n, f), 1.7)
    s["h"] = h.to(dt)
    s["stats"] = torch.stack(_norm_stats(s["a"].float(), kind, EPS) + _norm_stats(h, kind, EPS), 1)
    s["gx"], s["ga"], s["gt"] = torch.empty_like(s["h"]), torch.empty_like(s["a"]), empty(s["t"])
    for name in ("p", "p_bias", "s", "q", "q_bias"):
        s["g" + name] = empty(s[name])
    if case["bias"] is False:
        s["gp_bias"] = s["gq_bias"] = None
    return s


def _prepare_params(case, gen):
    sizes = _sizes(case)
    room = [_padded(n) for n in sizes]
    total, dt = sum(room), DTYPES[case["dtype"]]
    s = dict(case=case, max_norm=1.0)
    # every tensor lies at the start of its room in one stretch of memory; what pads it is zero
    held = torch.zeros(total, dtype=torch.bool, device="cuda")
    starts = [0]
    for r in room:
        starts.append(starts[-1] + r)
    for at, n in zip(starts, sizes):
        held[at:at + n] = True
    views = lambda flat: [flat[at:at + n] for at, n in zip(starts, sizes)]
    # gradients of a tensor have a size of their own, and its units differ among themselves
    scale = torch.exp(_normal(gen, (total,), 0.7)) * 1e-4
    s["g"] = _normal(gen, (total,)) * scale * held
    s["gs"] = views(s["g"])
    if case["op"] == NORM:
        s["out"] = torch.zeros(1, device="cuda")
        return s
    master = _normal(gen, (total,), 0.08) * held
    s["w"] = master.to(dt)
    s["ws"] = views(s["w"])
    s["master"] = s["w"].float() if case["master"] else None
    s["sq_norm"] = s["g"].double().square().sum().float().reshape(1)
    s["decays"] = _decays(case)
    s["decay"] = torch.repeat_interleave(torch.tensor(s["decays"], device="cuda"), torch.tensor([r // BLOCK for r in room], device="cuda"))
    m, v = _normal(gen, (total,), 0.3) * scale * held, (scale * (0.5 + torch.rand(total, generator=gen, device="cuda"))).square() * held * 1e-2
    s["scales"] = s["m_out"] = s["v_out"] = None
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
        return s
    mb, vb = m.view(-1, BLOCK), v.view(-1, BLOCK)
    s["scales"] = torch.stack([mb.abs().amax(1), vb.amax(1)], 1)
    tiny = torch.finfo(torch.float32).tiny
    s["m"] = torch.round(mb.sign() * (mb.abs() / s["scales"][:, :1].clamp_min(tiny)).sqrt() * 127).to(torch.int8).view(-1)
    s["v"] = torch.round((vb / s["scales"][:, 1:].clamp_min(tiny)).sqrt().sqrt() * 255).clamp_(0, 255).to(torch.uint8).view(-1)
    s["m_out"], s["v_out"] = torch.empty(total, dtype=torch.bfloat16, device="cuda"), torch.empty(total, dtype=torch.bfloat16, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (_prepare_rows if case["op"] in (FORWARD, BACKWARD) else _prepare_params)(case, gen)


# ---- the plain forms

def _plain_forward(s):
    kind, dt = s["case"]["norm"], s["a"].dtype

    def normed(z, gain, bias):
        mean, r = _norm_stats(z, kind, EPS)
        out = (z - mean[:, None]) * r[:, None] * gain
        return out if bias is None else out + bias

    y = normed(s["a"].float(), s["p"], s["p_bias"])
    branch = s["alpha"] * s["s"] * y
    if s["t"] is not None:
        branch = branch / (1 + torch.exp(-s["t"].float()))
    h = s["x"].float() + branch
    u = normed(h, s["q"], s["q_bias"]).to(dt)
    if s["hist"] is None:
        return {"h": h.to(dt), "u": u}
    s["hist"][s["idx"].long()] = u
    return {"h": h.to(dt), "u": u, "hist": s["hist"]}


def _plain_backward(s):
    layer, dt, f = s["case"]["norm"] == "layer", s["h"].dtype, s["case"]["width"]
    mean_a, r_a, mean_h, r_h = (c[:, None] for c in s["stats"].unbind(1))

    def through(d, z, r):
        out = d - z * ((d * z).sum(1, keepdim=True) / f)
        return r * (out - d.mean(1, keepdim=True) if layer else out)

    gu, hn = s["gu"].float(), (s["h"].float() - mean_h) * r_h
    e = s["gh"].float() + through(gu * s["q"], hn, r_h)
    an = (s["a"].float() - mean_a) * r_a
    y = an * s["p"] if s["p_bias"] is None else an * s["p"] + s["p_bias"]
    g = 1.0 if s["t"] is None else 1 / (1 + torch.exp(-s["t"].float()))
    ag = e * (s["alpha"] * g)
    dy = ag * s["s"]
    out = {"gx": e.to(dt), "ga": through(dy * s["p"], an, r_a).to(dt), "gq": (gu * hn).sum(0), "gp": (dy * an).sum(0), "gs": (ag * y).sum(0)}
    if s["t"] is not None:
        gt = dy * y * (1 - g)
        out["gt"] = (gt if s["case"]["gate"] == "full" else gt.sum(1, keepdim=True)).to(dt)
    if s["p_bias"] is not None:
        out["gq_bias"], out["gp_bias"] = gu.sum(0), dy.sum(0)
    return out


def _dice(total, device):
    """Two numbers of 16 bits for every element, from its place and the step's number."""
    x = torch.arange(total, dtype=torch.int64, device=device)
    x = ((x & 0xFFFFFFFF) + (x >> 32) * 0x85EBCA6B) & 0xFFFFFFFF
    x = x ^ (STEP * 0x9E3779B9 & 0xFFFFFFFF)
    x = (x ^ (x >> 16)) * 0x7FEB352D & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x846CA68B & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return x & 0xFFFF, x >> 16


def _coded(a, power, top, dice):
    """Scales and codes of non-negative values in blocks: value = scale * (code / top)^power, rounded at random to a neighbour."""
    blocks = a.view(-1, BLOCK)
    scale = blocks.amax(1, keepdim=True)
    scale = torch.where(scale >= torch.finfo(torch.float32).tiny, scale, torch.zeros_like(scale))
    x = blocks * torch.where(scale > 0, 1 / scale, torch.zeros_like(scale)) * float(top ** power)
    below = x.sqrt() if power == 2 else x.sqrt().sqrt()
    below = below.floor().clamp_max(top - 1)
    lower, upper = below.square(), (below + 1).square()
    lower, upper = (lower, upper) if power == 2 else (lower.square(), upper.square())
    up = (dice.view(-1, BLOCK).float() + 0.5) * (1 / 65536) * (upper - lower) < x - lower
    return scale, below + up


def _plain_adamw(s):
    eight, master = s["case"]["bits"] == 8, s["master"]
    c = (s["max_norm"] / (s["sq_norm"].sqrt() + 1e-6)).clamp_max(1.0)
    g = s["g"] * c
    if eight:
        k = s["m"].float()
        m = s["scales"][:, :1] * (k * k.abs() * (1 / 127 ** 2)).view(-1, BLOCK)
        k = s["v"].float().square().mul_(1 / 255 ** 2).view(-1, BLOCK)
        v = s["scales"][:, 1:] * k * k
        m, v = m.view(-1), v.view(-1)
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    w = master if master is not None else s["w"].float()
    denom = v.sqrt() * (1 / math.sqrt(1 - BETA2 ** STEP)) + ADAM_EPS
    w = w - (w.view(-1, BLOCK) * (LR * s["decay"])[:, None]).view(-1) - m * (LR / (1 - BETA1 ** STEP)) / denom
    s["w"].copy_(w)
    out = {"w": s["w"], "m": s["m"], "v": s["v"]}
    if master is not None:
        out["master"] = master.copy_(w)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return out
    dice = _dice(m.numel(), m.device)
    scale_m, km = _coded(m.abs(), 2, 127, dice[0])
    scale_v, kv = _coded(v, 4, 255, dice[1])
    kv = torch.where((kv == 0) & (v.view(-1, BLOCK) > 0) & (scale_v > 0), torch.ones_like(kv), kv)
    km = km * m.view(-1, BLOCK).sign()
    s["m"].copy_(km.view(-1))
    s["v"].copy_(kv.view(-1))
    s["scales"].copy_(torch.cat([scale_m, scale_v], 1))
    k = kv.square() * (1 / 255 ** 2)
    out["m"] = (scale_m * (km * km.abs() * (1 / 127 ** 2))).view(-1).to(torch.bfloat16)      # as many digits as 8 bits hold
    out["v"] = (scale_v * k * k).view(-1).to(torch.bfloat16)
    return out


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == NORM:
            return s["g"].square().sum().reshape(1)
        return {FORWARD: _plain_forward, BACKWARD: _plain_backward, ADAMW: _plain_adamw}[op](s)
    import paper_2106_05609_amd as gas
    if op == NORM:
        gas.gas_sq_norms(s["gs"], s["out"])
        return s["out"]
    if op == ADAMW:
        gas.gas_adamw_steps(s["ws"], s["gs"], s["m"], s["v"], LR, STEP, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=s["decays"],
                            scales=s["scales"], master=s["master"], sq_norm=s["sq_norm"], max_norm=s["max_norm"])
        out = {"w": s["w"], "m": s["m"], "v": s["v"]}
        if s["master"] is not None:
            out["master"] = s["master"]
        if s["scales"] is not None:
            gas.gas_adamw_unpack(s["m"], s["v"], s["scales"], s["m_out"], s["v_out"])
            out["m"], out["v"] = s["m_out"], s["v_out"]
        return out
    kind = KINDS[s["case"]["norm"]]
    same = dict(a=s["a"], t=s["t"], post=kind, p=s["p"], p_bias=s["p_bias"], s=s["s"], alpha=s["alpha"], pre=kind, q=s["q"])
    if op == FORWARD:
        gas.gas_residual_norm(s["x"], h=s["h"], u=s["u"], q_bias=s["q_bias"], eps=EPS, idx=s["idx"], hist=s["hist"], **same)
        return {k: s[k] for k in ("h", "u", "hist") if s[k] is not None}
    gas.gas_residual_norm_bwd(s["gh"], s["gu"], s["h"], s["stats"], s["gx"], ga=s["ga"], gt=s["gt"], gp=s["gp"], gp_bias=s["gp_bias"],
                              gs=s["gs"], gq=s["gq"], gq_bias=s["gq_bias"], **same)
    return {k: s[k] for k in ("gx", "ga", "gt", "gq", "gp", "gs", "gp_bias", "gq_bias") if s[k] is not None}


def work(case):
    if case["op"] in (FORWARD, BACKWARD):
        n, f, eb = case["rows"], case["width"], 4 if case["dtype"] == "f32" else 2
        gate = {"none": 0, "full": f, "row": 1}[case["gate"]]
        vectors = f * (5 if case["bias"] else 3) * 4
        if case["op"] == FORWARD:                  # x, a, t in; h, u out, u once more to the table
            return dict(bytes=eb * n * (4 * f + gate + (f if case["push"] else 0)) + (4 * n if case["push"] else 0) + vectors, flops=20 * n * f)
        return dict(bytes=eb * n * (6 * f + 2 * gate) + 16 * n + 2 * vectors, flops=40 * n * f)      # gh, gu, h, a, t in; gx, ga, gt out
    n, w = sum(_sizes(case)), 4 if case["dtype"] == "f32" else 2
    if case["op"] == NORM:
        return dict(bytes=4 * n, flops=2 * n)
    weights = w + 8 if case["master"] else 2 * w   # a master is read and written, the weights beside it are written
    states = 16 if case["bits"] == 32 else 2 * 2 + 4 + 16 / BLOCK                      # and what 8 bits stand for is written
    return dict(bytes=n * (weights + 4 + states), flops=15 * n)


# ---- the definitions in 64 bits

def _exact_forward(s):
    def norm(z):
        if s["case"]["norm"] == "layer":
            z = z - z.sum(1, keepdim=True) / z.shape[1]
        return z / (torch.linalg.vector_norm(z, dim=1, keepdim=True).square() / z.shape[1] + EPS).sqrt()
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    y = norm(d["a"]).mul_(d["p"]).add_(d.get("p_bias", 0.0))
    gate = torch.sigmoid(d["t"]) if "t" in d else 1.0
    h = torch.addcmul(d["x"], y.mul_(gate), d["s"], value=s["alpha"])
    u = norm(h).mul_(d["q"]).add_(d.get("q_bias", 0.0))
    if s["hist"] is None:
        return {"h": h, "u": u}
    return {"h": h, "u": u, "hist": d["hist"].index_copy(0, s["idx"].long(), u)}


def _exact_backward(s):
    """Each norm's Jacobian is symmetric, r (1 - P), P the projection on the normed row and, for a layer norm, on the row of ones;
    sums over the rows are products with a row of ones."""
    n, f = s["h"].shape
    d = {k: s[k].double() for k in ("gh", "gu", "h", "a", "stats", "p", "s", "q")}
    ones = torch.ones(1, n, dtype=torch.float64, device="cuda")
    over_rows = lambda z: torch.mv(z.t(), ones[0])

    def jacobian(z, row, r):
        along = torch.linalg.vecdot(z, row).div_(f)
        flat = z.mean(1) if s["case"]["norm"] == "layer" else torch.zeros_like(along)
        return torch.addcmul(z - flat[:, None], row, along[:, None], value=-1).mul_(r)

    unit_h = torch.sub(d["h"], d["stats"][:, 2:3]).mul_(d["stats"][:, 3:4])
    unit_a = torch.sub(d["a"], d["stats"][:, 0:1]).mul_(d["stats"][:, 1:2])
    out = {"gq": over_rows(d["gu"] * unit_h), "gx": d["gh"] + jacobian(d["gu"] * d["q"], unit_h, d["stats"][:, 3:4])}
    y = unit_a * d["p"]
    if s["p_bias"] is not None:
        y += s["p_bias"].double()
    gate = torch.ones((), dtype=torch.float64, device="cuda") if s["t"] is None else torch.sigmoid(s["t"].double())
    coefficient = s["alpha"] * gate * d["s"]                 # dh/dy
    out["gs"] = over_rows(out["gx"] * y * gate) * s["alpha"]
    out["gp"] = over_rows(out["gx"] * coefficient * unit_a)
    if s["p_bias"] is not None:
        out["gp_bias"], out["gq_bias"] = over_rows(out["gx"] * coefficient), over_rows(d["gu"])
    if s["t"] is not None:
        gt = out["gx"] * y * d["s"] * s["alpha"]
        gt = gt if s["case"]["gate"] == "full" else gt.sum(1, keepdim=True)
        out["gt"] = gt * gate * torch.sigmoid(-s["t"].double())
    out["ga"] = jacobian(out["gx"] * coefficient * d["p"], unit_a, d["stats"][:, 1:2])
    return out


def _exact_adamw(s):
    g = s["g"].double()
    g = g * min(1.0, s["max_norm"] / (math.sqrt(float(s["sq_norm"])) + 1e-6))
    per_block = lambda z: z.repeat_interleave(BLOCK)
    m, v = s["m"].double(), s["v"].double()
    if s["case"]["bits"] == 8:
        m = m.abs().mul_(m).div_(16129.0) * per_block(s["scales"][:, 0].double())
        v = v.div_(255.0).pow_(4) * per_block(s["scales"][:, 1].double())
    m, v = torch.lerp(g, m, BETA1), torch.lerp(g * g, v, BETA2)
    w = (s["w"] if s["master"] is None else s["master"]).double()
    step = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS)
    w = w * (1 - LR * per_block(s["decay"].double())) - LR * step
    out = {"w": w, "m": m, "v": v}
    if s["master"] is not None:
        out["master"] = w
    if s["case"]["bits"] == 32:
        return out
    places = _dice(m.numel(), m.device)
    for name, z, top, power, die in (("m", m, 127, 2, places[0]), ("v", v, 255, 4, places[1])):
        scale = per_block(z.abs().view(-1, BLOCK).amax(1))
        x = torch.where(scale > 0, z.abs() / scale, 0.0)
        low = (x.pow(1 / power) * top).floor().clamp_(0, top - 1)
        from_, to = (low / top).pow(power), ((low + 1) / top).pow(power)
        code = low + ((die.double() + 0.5) / 65536 < (x - from_) / (to - from_))
        if name == "v":
            code = torch.where((z > 0) & (code < 1), torch.ones_like(code), code)
        out[name] = z.sign() * scale * (code / top).pow(power)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == NORM:
        g = s["g"].double()
        return torch.dot(g, g).reshape(1)
    return {FORWARD: _exact_forward, BACKWARD: _exact_backward, ADAMW: _exact_adamw}[case["op"]](s)
