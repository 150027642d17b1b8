"""Output layers over many classes at sizes with at least 256 tiles of 256 rows by 256 classes, which workgroups take one after another: the loads of the next
tile begin, and its entries are fetched, while this one's logits are used; and at few rows of a large W. Against the definitions in 64 bits (tests/classes_reference.py), formed on the GPU."""
import math

import pytest
import torch

import paper_2106_05609_amd as gas
from tests import classes_reference as R
from tests.test_gpu_classes import DT, backward, check, distill_forward, exact_layer, forward, make, top, with_teacher

pytestmark = pytest.mark.gpu
# rows, width, classes: 705, 785 and 822 tiles; one step of 64 products, two, and several; W packed, W in place where it is bf16
SIZES = [(600, 20, 60_011), (1100, 70, 40_000), (520, 200, 70_016)]


def wide(t):
    return None if t is None else t.double() if t.is_floating_point() else t


def here(want):
    return tuple(v.cpu() for v in want)


def twice(call):
    """What a call leaves, and the same bits again over whatever the workspace holds then."""
    got = call()
    junk = torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda")
    del junk
    again = call()
    assert all(torch.equal(got[k], again[k]) for k in got)
    return got


@pytest.mark.parametrize("n, f, c", SIZES)
@pytest.mark.parametrize("dtype, gw", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("bias", [False, True])
def test_cross_entropy(n, f, c, dtype, gw, bias):
    s, gen = make(n, f, c, dtype, bias)
    row_scale = torch.randn(n, generator=gen).cuda()
    got = twice(lambda: forward(s))
    with torch.device("cuda"):
        x, w, b = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        want = R.xent(x, w, b, s["labels"])
        total = want["loss"][0].sum().reshape(1)
        want["sum"] = (total, want["loss"][1].sum() + 2 * R.U32 * total.abs())
        for name in got:
            check(got[name], here(want[name]), name)
        grads = twice(lambda: backward(s, got["lse"], dtype, gw, row_scale=row_scale))
        g, off = R.grad_at_logits(x, w, b, wide(got["lse"]), s["labels"], row_scale.double())
        for name, v in R.gradients(x, w, g, off, 0.37, dtype == "bf16", gw == "bf16").items():
            check(grads[name], here(v), name)


# temperature, labels, bias, entries next to each other (many of them in a tile), how many entries
DISTILL = [(1.0, False, True, True, 7), (2.0, True, True, True, 64), (1.5, True, False, True, 40), (2.0, False, False, False, 64), (1.0, True, True, False, 30),
           (3.0, True, True, True, 200)]


@pytest.mark.parametrize("n, f, c", SIZES)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t, labels, bias, near, k", DISTILL)
def test_distillation(n, f, c, dtype, t, labels, bias, near, k):
    s, gen = with_teacher(n, f, c, k, dtype, 0.6, near, bias=bias)
    row_scale = torch.randn(n, generator=gen).cuda()
    lab = s["labels"] if labels else None
    got = twice(lambda: distill_forward(s, t, 0.3, labels))

    def gradients():
        nan = lambda shape, dt=torch.float32: torch.full(shape, math.nan, dtype=dt, device="cuda")
        out = dict(gx=nan((n, f), DT[dtype]), gw=nan((f, c)), gbias=nan((c,)))
        gas.gas_linear_distill_bwd(s["x"], s["w"], s["ids"], s["values"], got["lse"], bias=s["bias"], labels=lab, temperature=t, label_weight=0.3, scale=0.6,
                                   row_scale=row_scale, **out)
        return out
    grads = twice(gradients)
    with torch.device("cuda"):
        x, w, b = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        want = R.distill(x, w, b, s["ids"], s["values"], t, lab, 0.3)
        check(got["loss"], here(want["loss"]), "loss")
        check(got["lse"], here(want["lse"]), "lse")
        g, off = R.grad_at_logits(x, w, b, wide(got["lse"]), lab, row_scale.double(), s["ids"], s["values"], t, 0.3)
        for name, v in R.gradients(x, w, g, off, 0.6, dtype == "bf16", False).items():
            check(grads[name], here(v), name)


# pieces of 4,096 classes, 28,672 and the rest; of the last size the first piece has 256 tiles
TOP = [(600, 16, 70_000, 64), (1100, 70, 40_001, 20), (300, 200, 100_000, 128), (4000, 30, 9000, 33)]


@pytest.mark.parametrize("n, f, c, k", TOP)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bias", [False, True])
def test_top_logits(n, f, c, k, dtype, bias):
    s = exact_layer(n, f, c, dtype, bias=bias)
    got = twice(lambda: top(s, k))
    with torch.device("cuda"):
        z = wide(s["x"]) @ wide(s["w"]) + (wide(s["bias"]) if bias else 0.0)
        ids, values = R.top(z, k)
        assert torch.equal(got["ids"].long(), ids) and torch.equal(got["values"].double(), values)
        check(got["lse"], here(R.log_sum_exp(z, torch.zeros_like(z))), "lse")


@pytest.mark.parametrize("dtype", list(DT))
def test_top_of_logits_in_hard_orders(dtype):
    """Rising with the class, falling, all equal, in blocks of equal ones, and with -infinity and NaN between."""
    n, c, k = 600, 70_000, 100
    x = torch.ones(n, 1, device="cuda", dtype=DT[dtype])
    at = torch.arange(c, device="cuda")
    for order in (at // 130, -(at // 130), at * 0, (at // 1000) % 7):
        s = dict(x=x, w=order[None].float().to(DT[dtype]), bias=None)
        got = top(s, k)
        ids, values = R.top(wide(s["w"]), k)
        assert (got["ids"] == ids).all() and (got["values"] == values).all()
    bias = torch.full((c,), -math.inf, device="cuda", dtype=DT[dtype])
    bias[::977], bias[5::1009], bias[60_000] = 2.0, math.nan, math.inf
    got = top(dict(s, bias=bias), k, lse=False)
    ids, values = R.top(wide(s["w"]) + wide(bias), k)
    assert (got["ids"] == ids).all() and torch.equal(got["values"].double(), values.expand(n, k))


@pytest.mark.parametrize("n, f, c", [(40, 600, 33_001), (64, 1100, 8001), (12, 64, 40_003), (33, 2048, 2047), (9, 300, 13_000), (64, 64, 32_769), (6, 600, 33_001)])
@pytest.mark.parametrize("dtype, gw", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_few_rows_and_a_large_w(n, f, c, dtype, gw):
    """W read once, in whole and in split sums, in place and copied: on both sides of where it is."""
    s, _ = make(n, f, c, dtype)
    got = twice(lambda: forward(s))
    with torch.device("cuda"):
        x, w, b = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        want = R.xent(x, w, b, s["labels"])
        for name in ("loss", "lse"):
            check(got[name], here(want[name]), name)
        grads = twice(lambda: backward(s, got["lse"], dtype, gw))
        g, off = R.grad_at_logits(x, w, b, wide(got["lse"]), s["labels"], None)
        for name, v in R.gradients(x, w, g, off, 0.37, dtype == "bf16", gw == "bf16").items():
            check(grads[name], here(v), name)
