"""The calls of an output layer over many classes against their definitions in 64 bits (tests/classes_reference.py, which derives
how far off they may be)."""
import math

import pytest
import torch

import paper_2106_05609_amd as gas
from tests import classes_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows, width, classes: one of everything, below and above a tile's sides, steps' and pieces' ends
SIZES = [(1, 1, 1), (1, 1, 2), (2, 3, 5), (3, 64, 255), (5, 17, 256), (64, 8, 257), (65, 33, 511), (63, 64, 512), (64, 65, 1000), (130, 100, 777),
         (255, 128, 264), (256, 129, 300), (257, 300, 513), (300, 1433, 264), (31, 2050, 97), (700, 40, 4001), (513, 256, 2056),
         (9, 1030, 600), (7, 1100, 700), (64, 2048, 263), (65, 700, 1000), (200, 1500, 2000)]


def mat(values, dtype, ld=None, off=0):
    """On the GPU as rows of stride ld from element `off` on; what is between the rows is NaN."""
    n, c = values.shape
    step = c if ld is None else ld
    flat = torch.full((off + max(1, n) * step + 64,), math.nan, dtype=DT[dtype], device="cuda")
    m = torch.as_strided(flat, (n, c), (step, 1), off)
    m.copy_(values.to(DT[dtype]))
    return m


def make(n, f, c, dtype, bias=True, seed=0, ld=(None, None), off=(0, 0), labelled=0.7, spread=1.5):
    gen = torch.Generator().manual_seed(seed + 31 * n + 7 * f + c)
    r = lambda *s: torch.randn(*s, generator=gen)
    s = dict(x=mat(r(n, f), dtype, ld[0], off[0]), w=mat(r(f, c) * spread / math.sqrt(f), dtype, ld[1], off[1]),
             bias=r(c).to(DT[dtype]).cuda() if bias else None)
    labels = torch.randint(0, c, (n,), generator=gen, dtype=torch.int32)
    none = torch.rand(n, generator=gen) >= labelled
    labels[none] = torch.tensor([-1, c, -7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(n) % 5][none]
    s["labels"] = labels.cuda()
    return s, gen


def wide(t):
    return None if t is None else t.double().cpu() if t.is_floating_point() else t.cpu()


def check(got, want, what):
    value, off = want
    got = got.double().cpu()
    assert got.shape == value.shape, what
    same = (got == value) | (got.isnan() & value.isnan())
    worst = torch.where(same, 0.0, (got - value).abs() / (off + 1e-30))
    worst = worst.nan_to_num(nan=math.inf).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (what, worst)


def forward(s, **kw):
    n = s["x"].shape[0]
    out = dict(loss=torch.full((n,), 9.0, device="cuda"), lse=torch.full((n,), 9.0, device="cuda"), sum=torch.full((1,), 9.0, device="cuda"))
    gas.gas_linear_xent(s["x"], s["w"], s["labels"], out["loss"], out["lse"], bias=s["bias"], loss_sum=out["sum"], **kw)
    return out


def backward(s, lse, dtype, gw="f32", scale=0.37, row_scale=None, **kw):
    c = s["w"].shape[1]
    nan = lambda shape, dt: torch.full(shape, math.nan, dtype=DT[dt], device="cuda")
    out = dict(gx=nan(s["x"].shape, dtype), gw=nan(s["w"].shape, gw), gbias=nan((c,), "f32"))
    gas.gas_linear_xent_bwd(s["x"], s["w"], s["labels"], lse, bias=s["bias"], scale=scale, row_scale=row_scale, **out, **kw)
    return out


def close(a, b):
    """Relative error of all of it."""
    b = b.double()
    return ((a.double().cpu() - b.cpu()).norm() / b.cpu().norm().clamp_min(1e-300)).item()


@pytest.mark.parametrize("n, f, c", SIZES)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bias", [False, True])
def test_cross_entropy(n, f, c, dtype, bias):
    s, _ = make(n, f, c, dtype, bias)
    got = forward(s)
    want = R.xent(wide(s["x"]), wide(s["w"]), wide(s["bias"]), wide(s["labels"]))
    check(got["loss"], want["loss"], "loss")
    check(got["lse"], want["lse"], "lse")
    total = want["loss"][0].sum().reshape(1)
    check(got["sum"], (total, want["loss"][1].sum() + 2 * R.U32 * total.abs()), "sum")


@pytest.mark.parametrize("n, f, c", SIZES)
@pytest.mark.parametrize("dtype, gw", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("weighted", [False, True])
def test_cross_entropy_backward(n, f, c, dtype, gw, weighted):
    s, gen = make(n, f, c, dtype)
    row_scale = torch.randn(n, generator=gen).cuda() if weighted else None
    lse = forward(s)["lse"]
    got = backward(s, lse, dtype, gw, row_scale=row_scale)
    x, w = wide(s["x"]), wide(s["w"])
    g, off = R.grad_at_logits(x, w, wide(s["bias"]), wide(lse), wide(s["labels"]), wide(row_scale))
    for name, want in R.gradients(x, w, g, off, 0.37, dtype == "bf16", gw == "bf16").items():
        check(got[name], want, name)


@pytest.mark.parametrize("rows", [40, 300])
def test_sums_in_fp32_keep_their_digits(rows):
    """Errors of sums of k terms of random signs grow as the root of k: (12 + sqrt(k)) u of all of it, a third of which is expected; a product
    without the operands' third parts would be off by 2^-17, more than this for every k here."""
    n, f, c = rows, 250, 2900
    s, _ = make(n, f, c, "f32", labelled=1.0)
    lse = forward(s)["lse"]
    got = backward(s, lse, "f32")
    x, w = wide(s["x"]), wide(s["w"])
    g, _ = R.grad_at_logits(x, w, wide(s["bias"]), wide(lse), wide(s["labels"]), None)
    want = R.gradients(x, w, g, g * 0, 0.37, False, False)
    for name, k in (("gx", c), ("gw", n)):
        assert close(got[name], want[name][0]) <= R.U32 * (12 + math.sqrt(k)), name


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("ld, off", [((40, 304), (0, 0)), ((41, 301), (1, 3)), ((37, 312), (8, 4)), ((200, 1000), (5, 8))])
def test_strides_and_alignments(dtype, ld, off):
    n, f, c = 140, 37, 296
    s, _ = make(n, f, c, dtype, ld=ld, off=off)
    plain, _ = make(n, f, c, dtype)
    got, want = forward(s), forward(plain)
    lse = want["lse"]
    for name in got:
        assert torch.equal(got[name], want[name]), name
    grads = backward(plain, lse, dtype)
    gx, gw = mat(torch.zeros(n, f), dtype, ld[0], off[0]), mat(torch.zeros(f, c), "f32", ld[1], off[1])
    around = [(m, torch.as_strided(m, (n if m is gx else f, l - m.shape[1]), (l, 1), m.storage_offset() + m.shape[1])) for m, l in ((gx, ld[0]), (gw, ld[1]))]
    gas.gas_linear_xent_bwd(s["x"], s["w"], s["labels"], lse, gx=gx, gw=gw, bias=s["bias"], scale=0.37)
    assert torch.equal(gx, grads["gx"]) and torch.equal(gw, grads["gw"])
    assert all(between.isnan().all() for _, between in around)           # what is between the rows stays


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n", [1, 2, 4, 7])
@pytest.mark.parametrize("ld, off", [((40, 304), (0, 0)), ((41, 301), (1, 3)), ((200, 1000), (5, 8))])
def test_few_rows_of_any_alignment(dtype, n, ld, off):
    s, _ = make(n, 37, 296, dtype, ld=ld, off=off, labelled=1.0)
    plain, _ = make(n, 37, 296, dtype, labelled=1.0)
    got, want = forward(s), forward(plain)
    assert all(torch.equal(got[k], want[k]) for k in got)
    got, want = (backward(v, want["lse"], dtype) for v in (s, plain))
    assert all(torch.equal(got[k], want[k]) for k in got)


@pytest.mark.parametrize("n", [8, 40])
@pytest.mark.parametrize("dtype, gw", [("f32", "f32"), ("bf16", "bf16")])
def test_few_rows_of_more_classes_than_a_piece_has(dtype, gw, n):
    """2^21 of them are a piece where the rows are at most 256."""
    s, _ = make(n, 2, 2 ** 21 + 300, dtype)
    lse = forward(s)["lse"]
    got = backward(s, lse, dtype, gw)
    x, w = wide(s["x"]), wide(s["w"])
    g, off = R.grad_at_logits(x, w, wide(s["bias"]), wide(lse), wide(s["labels"]), None)
    for name, want in R.gradients(x, w, g, off, 0.37, dtype == "bf16", gw == "bf16").items():
        check(got[name], want, name)


@pytest.mark.parametrize("c", [2_100_000, 2_100_001])
@pytest.mark.parametrize("n", [3, 40, 300])
def test_offsets_beyond_32_bits(n, c):
    """W and its gradient of 2.3 G elements, zero but for nine classes: what those nine have to be follows from them alone."""
    f, gen = 1100, torch.Generator().manual_seed(n)
    at = torch.tensor([0, 5, 256, 70_001, 1_048_577, 2_000_000, 2_097_152, c - 2, c - 1])
    w = torch.zeros((f, c), dtype=torch.bfloat16, device="cuda")
    w[:, at.cuda()] = (torch.randn(f, 9, generator=gen) * 3 / math.sqrt(f)).bfloat16().cuda()
    pick = torch.randint(0, 9, (n,), generator=gen)
    s = dict(x=torch.randn(n, f, generator=gen).bfloat16().cuda(), w=w, bias=None, labels=at[pick].int().cuda())
    got = forward(s)
    x, few = wide(s["x"]), wide(w[:, at.cuda()])
    z, off = R.logits(x, few, None)
    lse = torch.log(torch.exp(z).sum(1) + (c - 9))
    off_lse = off.amax(1) + R.U32 * (120 + c / 256 / 16 + 8 * lse.abs() + 8 * z.abs().amax(1))
    check(got["lse"], (lse, off_lse), "lse")
    loss = lse - z.gather(1, pick[:, None])[:, 0]
    check(got["loss"], (loss, off_lse + off.amax(1) + 2 * R.U32 * loss.abs()), "loss")
    grads = dict(gx=torch.full_like(s["x"], math.nan), gw=torch.full_like(w, math.nan), gbias=torch.full((c,), math.nan, device="cuda"))
    gas.gas_linear_xent_bwd(s["x"], w, s["labels"], got["lse"], scale=0.37, **grads)
    g, off = R.grad_at_logits(x, few, None, wide(got["lse"]), pick.int(), None)
    for name, want in R.gradients(x, few, g, off, 0.37, True, True).items():
        check(grads[name] if name == "gx" else grads[name][..., at.cuda()], want, name)
    assert not any(v.isnan().any() for v in grads.values())


@pytest.mark.parametrize("dtype", list(DT))
def test_any_gradient_alone(dtype):
    s, _ = make(150, 70, 600, dtype)
    lse = forward(s)["lse"]
    every = backward(s, lse, dtype)
    for name in every:
        one = torch.full_like(every[name], math.nan)
        gas.gas_linear_xent_bwd(s["x"], s["w"], s["labels"], lse, bias=s["bias"], scale=0.37, **{name: one})
        assert torch.equal(one, every[name])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n", [6, 50, 270])
def test_rows_without_a_label(dtype, n):
    """NaN and infinities in them reach nothing; none labelled at all gives zeros."""
    s, _ = make(n, 70, 600, dtype, labelled=0.5)
    clean = forward(s)
    grads = backward(s, clean["lse"], dtype)
    off = (s["labels"] < 0) | (s["labels"] >= 600)
    assert 0 < int(off.sum()) < n
    s["x"][off] = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(DT[dtype]).repeat(200)[:70]
    lse = clean["lse"].clone()
    lse[off] = math.nan
    dirty, again = forward(s), backward(s, lse, dtype)
    assert all(torch.equal(clean[k], dirty[k]) for k in clean)
    assert all(torch.equal(grads[k], again[k]) for k in grads)
    assert (again["gx"][off] == 0).all()
    s["labels"].fill_(-1)
    none, zero = forward(s), backward(s, lse, dtype)
    assert all((v == 0).all() for v in (*none.values(), *zero.values()))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("low", [-math.inf, "least"])
@pytest.mark.parametrize("n, f", [(90, 20), (6, 20), (90, 1100)])
def test_classes_taken_out_by_the_bias(dtype, low, n, f):
    """-infinity, or the type's least value: probability 0, and a label on one an infinite (a very large) loss with a finite gradient.  A whole
    tile of them, and all but one."""
    c = 700
    low = torch.finfo(DT[dtype]).min if low == "least" else low
    for out in (slice(3, 9), slice(256, 512), slice(1, c)):
        s, _ = make(n, f, c, dtype, labelled=1.0)
        s["bias"][out] = low
        s["labels"][:] = 0
        s["labels"][5] = 300 if out != slice(3, 9) else 4
        got = forward(s)
        x, w, bias = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        want = R.xent(x, w, bias, wide(s["labels"]))
        check(got["lse"], want["lse"], "lse")
        rows = torch.arange(n) != 5
        check(got["loss"][rows.cuda()], (want["loss"][0][rows], want["loss"][1][rows]), "loss")
        assert got["loss"][5].item() > 1e37
        grads = backward(s, got["lse"], dtype)
        g, off = R.grad_at_logits(x, w, bias, wide(got["lse"]), wide(s["labels"]), None)
        for name, v in R.gradients(x, w, g, off, 0.37, dtype == "bf16", False).items():
            check(grads[name], v, name)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shift", [0.0, 80.0, -3000.0])
@pytest.mark.parametrize("n, f", [(70, 64), (7, 64), (70, 1100)])
def test_large_logits(dtype, shift, n, f):
    """Logits of some thousand, differences of some hundred: exponentials from the largest on."""
    c = 520
    s, _ = make(n, f, c, dtype, spread=60.0)
    s["bias"].add_(shift)
    got = forward(s)
    want = R.xent(wide(s["x"]), wide(s["w"]), wide(s["bias"]), wide(s["labels"]))
    check(got["lse"], want["lse"], "lse")
    check(got["loss"], want["loss"], "loss")


@pytest.mark.parametrize("n, f", [(80, 40), (8, 40), (80, 1100)])
def test_a_nan_in_a_row_stays_there(n, f):
    for dtype in DT:
        s, _ = make(n, f, 300, dtype, labelled=1.0)
        clean = forward(s)
        s["x"][7, 3] = math.nan
        got = forward(s)
        rows = torch.arange(n, device="cuda") != 7
        assert got["loss"][7].isnan() and got["lse"][7].isnan() and got["sum"].isnan().all()
        assert torch.equal(got["loss"][rows], clean["loss"][rows])
        grads = backward(s, got["lse"], dtype)
        assert grads["gx"][7].isnan().all() and not grads["gx"][rows].isnan().any()


def test_gradients_against_differences():
    """(loss(v + h) - loss(v - h)) / 2h in one element each of X, W and the bias, in fp32: the loss's sum of 40 terms of about 7 is off by some
    2e-5 in either call and h = 2^-5, so 2e-3 allows for that and for the third derivative's h^2 / 6."""
    s, _ = make(40, 24, 900, "f32", labelled=0.8)
    got = forward(s)
    grads = backward(s, got["lse"], "f32", scale=1.0)
    h = 2.0 ** -5
    label = int(s["labels"][s["labels"] >= 0][0])
    for key, at, name in (("x", (3, 5), "gx"), ("x", (0, 23), "gx"), ("w", (4, label), "gw"), ("w", (9, 899), "gw"), ("bias", (label,), "gbias")):
        sums = []
        for sign in (1, -1):
            t = dict(s, **{key: s[key].clone()})
            t[key][at] += sign * h
            sums.append(forward(t)["loss"].double().sum().item())
        assert abs((sums[0] - sums[1]) / (2 * h) - grads[name][at].item()) <= 2e-3, (key, at)


def test_empty_batch():
    x, w = torch.empty(0, 12, device="cuda"), torch.randn(12, 30, device="cuda")
    e, gw, gb, total = torch.empty(0, device="cuda"), torch.full((12, 30), 5.0, device="cuda"), torch.full((30,), 5.0, device="cuda"), torch.full((1,), 5.0, device="cuda")
    labels = torch.empty(0, dtype=torch.int32, device="cuda")
    gas.gas_linear_xent(x, w, labels, e, e.clone(), loss_sum=total)
    assert total.item() == 0
    gas.gas_linear_xent_bwd(x, w, labels, e, gx=torch.empty_like(x), gw=gw, gbias=gb)
    assert (gw == 0).all() and (gb == 0).all()
    ids, values = torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda")
    gas.gas_linear_top(x, w, ids, values)
    total.fill_(5.0)
    gw.fill_(5.0)
    gas.gas_linear_distill(x, w, ids, values, e, torch.empty(0, 2, device="cuda"), loss_sum=total)
    gas.gas_linear_distill_bwd(x, w, ids, values, torch.empty(0, 2, device="cuda"), gw=gw)
    assert total.item() == 0 and (gw == 0).all()


@pytest.mark.parametrize("dtype", list(DT))
def test_pieces_of_the_classes(dtype):
    """More gradients at the logits than there is room for: several pieces, of which the last is narrower; and with few rows that count the same
    call takes them in one."""
    n, f, c = 6500, 40, 100_001
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.randn(n, f, generator=gen, device="cuda").to(DT[dtype]), (torch.randn(f, c, generator=gen, device="cuda") * 0.2).to(DT[dtype])
    labels = torch.randint(0, c, (n,), generator=gen, device="cuda", dtype=torch.int32)
    for few in (False, True):
        if few:
            labels[torch.randperm(n, generator=gen, device="cuda")[40:]] = -1
        s = dict(x=x, w=w, bias=None, labels=labels)
        got = forward(s)
        grads = backward(s, got["lse"], dtype)
        on = (labels >= 0)[:, None]
        z = x.double() @ w.double()
        assert close(got["lse"], (torch.logsumexp(z, 1) * on[:, 0])) <= 16 * R.U32
        g = torch.exp(z.sub_(got["lse"].double()[:, None])).mul_(on)
        g.scatter_add_(1, labels.clamp(min=0).long()[:, None], -on.double())
        g.mul_(0.37)
        del z
        # bf16: the gradient at the logits and the result round by up to 2^-8, root mean square less than half of that each
        most = {"gx": (c, R.U16), "gw": (n, 0.75 * R.U16), "gbias": (n, 0)}
        for name, want in (("gx", g @ w.double().t()), ("gw", x.double().t() @ g), ("gbias", g.sum(0))):
            k, half = most[name]
            assert close(grads[name], want) <= R.U32 * (12 + math.sqrt(k)) + (half if dtype == "bf16" else 0), (name, few)


@pytest.mark.parametrize("n, f, c", [(400, 100, 3000), (6, 100, 3000), (30, 100, 3000), (100, 1100, 700)])
def test_the_same_bits_again(n, f, c):
    for dtype in DT:
        s, _ = make(n, f, c, dtype)
        first = forward(s)
        grads = backward(s, first["lse"], dtype)
        for _ in range(2):
            junk = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")     # what a workspace may hold before
            del junk
            again = forward(s)
            assert all(torch.equal(first[k], again[k]) for k in first)
            more = backward(s, first["lse"], dtype)
            assert all(torch.equal(grads[k], more[k]) for k in grads)


# ---- distillation

def with_teacher(n, f, c, k, dtype, labelled, near=False, seed=0, **kw):
    s, gen = make(n, f, c, dtype, seed=seed, labelled=labelled, **kw)
    if near and c >= k:                                   # all in one or two tiles, distinct
        ids = (torch.randint(0, c, (n, 1), generator=gen) + torch.rand(n, k, generator=gen).argsort(1)) % c
    else:
        ids = torch.randint(0, c, (n, k), generator=gen)                # some twice
    absent = torch.rand(n, k, generator=gen) < 0.15
    ids[absent] = torch.tensor([-1, c, -2 ** 31, 2 ** 31 - 1])[torch.arange(n * k).view(n, k) % 4][absent]
    values = torch.randn(n, k, generator=gen) * 3 + 20.0
    gone = torch.rand(n, k, generator=gen) < 0.05
    values[gone] = -math.inf
    values[absent] = math.nan
    if n > 2:
        ids[1], ids[2] = -1, -1                           # rows without any entry
    s["ids"], s["values"] = ids.to(torch.int32).cuda(), values.cuda()
    return s, gen


def distill_forward(s, t, label_weight, labels=True):
    n = s["x"].shape[0]
    out = dict(loss=torch.full((n,), 9.0, device="cuda"), lse=torch.full((n, 2), 9.0, device="cuda"), sum=torch.full((1,), 9.0, device="cuda"))
    gas.gas_linear_distill(s["x"], s["w"], s["ids"], s["values"], out["loss"], out["lse"], bias=s["bias"], labels=s["labels"] if labels else None,
                           temperature=t, label_weight=label_weight, loss_sum=out["sum"])
    return out


CASES = [(1, 4, 6, 1, 1.0, 0.5), (3, 5, 9, 4, 2.0, 0.3), (40, 33, 300, 7, 0.5, 0.0), (64, 64, 513, 64, 1.0, 1.0), (70, 20, 1000, 65, 3.0, 0.25),
         (300, 65, 700, 100, 2.0, 0.5), (257, 128, 2600, 256, 1.0, 0.4), (20, 300, 4001, 255, 4.0, 0.9), (50, 900, 700, 30, 2.0, 0.5), (130, 1100, 520, 40, 1.5, 0.5)]


@pytest.mark.parametrize("n, f, c, k, t, label_weight", CASES)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("labels", [False, True])
@pytest.mark.parametrize("near", [False, True])
def test_distillation(n, f, c, k, t, label_weight, dtype, labels, near):
    s, gen = with_teacher(n, f, c, k, dtype, 0.6, near)
    got = distill_forward(s, t, label_weight, labels)
    x, w, bias, lab = wide(s["x"]), wide(s["w"]), wide(s["bias"]), wide(s["labels"]) if labels else None
    ids, values = s["ids"].cpu(), s["values"].cpu()
    want = R.distill(x, w, bias, ids, values, t, lab, label_weight)
    check(got["loss"], want["loss"], "loss")
    check(got["lse"], want["lse"], "lse")
    row_scale = torch.randn(n, generator=gen).cuda()
    nan = lambda like, dt=None: torch.full(like.shape, math.nan, dtype=dt or like.dtype, device="cuda")
    grads = dict(gx=nan(s["x"]), gw=nan(s["w"], torch.float32), gbias=nan(s["bias"], torch.float32))
    gas.gas_linear_distill_bwd(s["x"], s["w"], s["ids"], s["values"], got["lse"], bias=s["bias"], labels=s["labels"] if labels else None, temperature=t,
                               label_weight=label_weight, scale=0.6, row_scale=row_scale, **grads)
    g, off = R.grad_at_logits(x, w, bias, wide(got["lse"]), lab, wide(row_scale), ids, values, t, label_weight)
    for name, v in R.gradients(x, w, g, off, 0.6, dtype == "bf16", False).items():
        check(grads[name], v, name)


def test_distillation_of_strided_entries():
    s, _ = with_teacher(90, 30, 400, 9, "f32", 0.5)
    want = distill_forward(s, 2.0, 0.5)
    ids, values = torch.full((90, 20), 3, dtype=torch.int32, device="cuda"), torch.full((90, 33), 2.0, device="cuda")
    ids[:, 4:13], values[:, 7:16] = s["ids"], s["values"]
    got = distill_forward(dict(s, ids=ids[:, 4:13], values=values[:, 7:16]), 2.0, 0.5)
    assert all(torch.equal(got[k], want[k]) for k in got)


def test_distillation_from_one_entry_is_cross_entropy():
    """T = 1 and all of the teacher's weight on one class."""
    for dtype in DT:
        s, _ = make(100, 50, 1200, dtype, labelled=0.8)
        bad = (s["labels"] < 0) | (s["labels"] >= 1200)
        s["ids"], s["values"] = torch.where(bad, -1, s["labels"])[:, None].contiguous(), torch.full((100, 1), 3.0, device="cuda")
        one, other = forward(s), distill_forward(s, 1.0, 0.5, labels=False)
        assert torch.allclose(one["loss"], other["loss"], rtol=4 * R.U32, atol=0) and torch.equal(one["lse"], other["lse"][:, 0])


def test_a_student_like_its_teacher_has_no_gradient():
    """Every class among the entries and the student's own logits in them: G = p - q is what rounding leaves."""
    s, _ = make(50, 32, 60, "f32")
    z = (wide(s["x"]) @ wide(s["w"]) + wide(s["bias"]))
    s["ids"] = torch.arange(60, dtype=torch.int32).repeat(50, 1).cuda()
    s["values"] = z.float().cuda()
    got = distill_forward(s, 2.0, 0.5, labels=False)
    assert got["loss"].abs().max().item() <= 4 * 200 * R.U32 * 8
    gx = torch.empty_like(s["x"])
    gas.gas_linear_distill_bwd(s["x"], s["w"], s["ids"], s["values"], got["lse"], gx=gx, bias=s["bias"], temperature=2.0)
    assert gx.abs().max().item() <= 2 * 60 * R.U32 * 100


# ---- the top logits

def exact_layer(n, f, c, dtype, seed=0, bias=True):
    """Values in steps: every sum of products is exact in fp32, so equal logits are equal and the order is known."""
    gen = torch.Generator().manual_seed(seed + n + f + c)
    step = lambda *shape: torch.randint(-6, 7, shape, generator=gen).float()
    return dict(x=step(n, f).div(4).to(DT[dtype]).cuda(), w=step(f, c).div(8).to(DT[dtype]).cuda(),
                bias=step(c).div(2).to(DT[dtype]).cuda() if bias else None)


def top(s, k, lse=True):
    n = s["x"].shape[0]
    out = dict(ids=torch.full((n, k), -5, dtype=torch.int32, device="cuda"), values=torch.full((n, k), math.nan, device="cuda"),
               lse=torch.full((n,), math.nan, device="cuda"))
    gas.gas_linear_top(s["x"], s["w"], out["ids"], out["values"], lse=out["lse"] if lse else None, bias=s["bias"])
    return out


@pytest.mark.parametrize("n, f, c, k", [(1, 1, 1, 1), (1, 3, 7, 7), (2, 8, 128, 128), (5, 2, 256, 10), (1, 64, 5000, 50), (9, 30, 4096, 128), (64, 40, 4097, 1),
                                        (65, 16, 9000, 64), (300, 2, 20_000, 100), (31, 1, 30_001, 128), (8, 300, 12_289, 17), (16, 100, 4100, 33),
                                        (17, 100, 4100, 33), (2, 512, 100_003, 10), (700, 33, 6001, 20), (20, 2048, 2000, 40), (100, 1000, 700, 64),
                                        (100, 800, 9000, 64)])
@pytest.mark.parametrize("dtype", list(DT))
def test_top_logits(n, f, c, k, dtype):
    s = exact_layer(n, f, c, dtype)
    got = top(s, k)
    z = wide(s["x"]) @ wide(s["w"]) + wide(s["bias"])
    ids, values = R.top(z, k)
    assert torch.equal(got["ids"].cpu().long(), ids)
    assert torch.equal(got["values"].cpu().double(), values)
    lse, off = R.log_sum_exp(z, torch.zeros_like(z))
    check(got["lse"], (lse, off), "lse")
    again = top(s, k, lse=False)
    assert torch.equal(again["ids"], got["ids"]) and again["lse"].isnan().all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n", [1, 7, 80])
def test_top_of_logits_in_hard_orders(dtype, n):
    """Rising with the class (each piece replaces the list), falling, all equal, and in blocks of equal ones."""
    c, k = 33_000, 128
    x = torch.ones(n, 1, device="cuda", dtype=DT[dtype])
    at = torch.arange(c)
    for order in (at // 130, -(at // 130), at * 0, (at // 1000) % 7, -(at == c - 1).long()):
        s = dict(x=x, w=order[None].float().to(DT[dtype]).cuda(), bias=None)
        got = top(s, k)
        ids, values = R.top(wide(s["w"]).expand(n, c), k)
        assert torch.equal(got["ids"].cpu().long(), ids) and torch.equal(got["values"].cpu().double(), values)


@pytest.mark.parametrize("n", [3, 90])
def test_top_with_infinities_and_nan(n):
    """-infinity is below every number and above NaN; rows with little else name those too."""
    c, k = 9000, 40
    for dtype in DT:
        s = exact_layer(n, 3, c, dtype)
        s["bias"][:] = -math.inf
        keep = torch.tensor([5, 4500, 8999], device="cuda")
        s["bias"][keep] = 1.0
        s["bias"][torch.tensor([0, 17, 5000], device="cuda")] = math.nan
        s["bias"][6000] = math.inf
        got = top(s, k, lse=False)
        z = wide(s["x"]) @ wide(s["w"]) + wide(s["bias"])
        ids, values = R.top(z, k)
        assert torch.equal(got["ids"].cpu().long(), ids) and torch.equal(got["values"].cpu().double(), values)
        s["bias"][:] = math.nan
        got = top(s, k)
        assert torch.equal(got["ids"].cpu().long(), torch.arange(k).expand(n, k)) and got["values"].isnan().all() and got["lse"].isnan().all()


def test_top_of_strided_outputs():
    s = exact_layer(20, 8, 500, "f32")
    ids, values = torch.full((20, 9), -5, dtype=torch.int32, device="cuda"), torch.full((20, 11), math.nan, device="cuda")
    want = top(s, 6)
    gas.gas_linear_top(s["x"], s["w"], ids[:, 2:8], values[:, 4:10], bias=s["bias"])
    assert torch.equal(ids[:, 2:8], want["ids"]) and torch.equal(values[:, 4:10], want["values"])
    assert (ids[:, [0, 1, 8]] == -5).all() and values[:, [0, 1, 2, 3, 10]].isnan().all()


# ---- together

@pytest.mark.parametrize("n, f, c", [(200, 64, 3000), (5, 64, 3000), (30, 64, 3000), (100, 1100, 700)])
def test_on_another_stream_and_in_graphs(n, f, c):
    """A forward and a backward call in one graph, the top logits in another, replayed in turn with eager work between, on inputs that change."""
    for dtype in DT:
        s, _ = with_teacher(n, f, c, 12, dtype, 0.5)
        out = dict(loss=torch.empty(n, device="cuda"), lse=torch.empty(n, 2, device="cuda"))
        grads = dict(gx=torch.empty_like(s["x"]), gw=torch.empty(f, c, device="cuda"), gbias=torch.empty(c, device="cuda"))
        ids, values, lse = torch.empty(n, 5, dtype=torch.int32, device="cuda"), torch.empty(n, 5, device="cuda"), torch.empty(n, device="cuda")
        work = torch.empty(max(gas.gas_linear_distill_workspace(n, f, c, DT[dtype], 12), gas.gas_linear_distill_bwd_workspace(n, f, c, DT[dtype], 12),
                               gas.gas_linear_top_workspace(n, f, c, DT[dtype], 5)), dtype=torch.uint8, device="cuda")
        same = dict(bias=s["bias"], labels=s["labels"], temperature=2.0, label_weight=0.3, workspace=work)

        def train():
            gas.gas_linear_distill(s["x"], s["w"], s["ids"], s["values"], out["loss"], out["lse"], **same)
            gas.gas_linear_distill_bwd(s["x"], s["w"], s["ids"], s["values"], out["lse"], **grads, **same)

        def answer():
            gas.gas_linear_top(s["x"], s["w"], ids, values, lse=lse, bias=s["bias"], workspace=work)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs = []
        with torch.cuda.stream(side):
            for call in (train, answer):
                call()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    call()
                graphs.append(g)
        torch.cuda.current_stream().wait_stream(side)
        every = (*out.values(), *grads.values(), ids, values, lse)
        for turn in range(4):
            s["x"].mul_(-0.9)
            s["w"].add_(0.01)
            if turn % 2:
                s["labels"][turn::3] = 7
            train()
            answer()
            want = [t.clone() for t in every]
            for t in every:
                t.zero_()
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(every, want))


def test_a_teacher_and_its_student():
    """The teacher's top logits as they come out are what the student is trained from; with all of the teacher's classes kept and T = 1 the
    loss is the divergence of the two distributions."""
    t, _ = make(120, 48, 128, "f32", seed=1)
    s, _ = make(120, 32, 128, "f32", seed=2)
    got = top(t, 128)
    z_t = wide(t["x"]) @ wide(t["w"]) + wide(t["bias"])
    z_s = wide(s["x"]) @ wide(s["w"]) + wide(s["bias"])
    s.update(ids=got["ids"], values=got["values"])
    loss = distill_forward(s, 1.0, 0.5, labels=False)["loss"]
    log_q, log_p = torch.log_softmax(z_t, 1), torch.log_softmax(z_s, 1)
    want = (log_q.exp() * (log_q - log_p)).sum(1)
    assert (loss.double().cpu() - want).abs().max().item() <= 2000 * R.U32
