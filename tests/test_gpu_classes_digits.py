"""Digits of the products of an output layer over many classes on every path that its sizes choose, and ties between classes that different launches form."""
import math

import pytest
import torch

import paper_2106_05609_amd as gas
from tests import classes_reference as R
from tests.test_gpu_classes import DT, backward, check, close, exact_layer, forward, make, top

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n, f, half", [(100, 1000, 4096), (70, 300, 4096), (600, 512, 4096), (2, 1100, 4096), (40, 1000, 4096), (1000, 40, 4096), (300, 300, 35_000),
                                        (300, 70, 35_000), (100, 1000, 2000)])
def test_equal_logits_of_classes_far_apart(n, f, half, dtype, bias):
    """Every class twice, the second time in another piece or another kind of tile: two and two equal, the lower one first, however their sums are formed."""
    k = 64
    s, _ = make(n, f, half, dtype, bias)
    s["w"] = torch.cat([s["w"], s["w"]], 1)
    if bias:
        s["bias"] = torch.cat([s["bias"], s["bias"]])
    got = top(s, k)
    ids, values = got["ids"], got["values"]
    fell, same = values[:, :-1] > values[:, 1:], values[:, :-1] == values[:, 1:]
    assert (fell | (same & (ids[:, :-1] < ids[:, 1:]))).all()
    # above the last value both of every pair are there, and equal
    whole = values > values[:, -1:]
    pair = (ids % half)[:, :, None] == (ids % half)[:, None, :]
    assert (pair.sum(2)[whole] == 2).all() and not (pair & (values[:, :, None] != values[:, None, :])).any()


def most_off(k, own=1.0):
    """Of a sum of k fp32 products, relative and as a root mean square over many sums: the last rounding and `own` units beside; k / 16 roundings to half a step at most, evenly
    spread (a third of its square), of a sum that grows to its size as its terms' squares do (half of that), of which half as much again is allowed."""
    return R.U32 * (own + 1.5 * math.sqrt(k / 16 / 6))


def two_parts(a):
    """What is left of fp32 values without the third of their bf16 parts."""
    high = a.float().bfloat16().float()
    return (high + (a.float() - high).bfloat16().float()).double()


# the vector units; few rows in split sums; W read as it lies, in whole sums and in split ones; small tiles, whole and split; many tiles
PATHS = [(5, 250, 2900), (6, 1100, 2900), (40, 200, 2900), (40, 250, 2900), (200, 200, 2900), (200, 300, 2900), (300, 200, 40_000)]


@pytest.mark.parametrize("n, f, c", PATHS + [(5, 2048, 66_000), (40, 2048, 66_000), (100, 2048, 66_000), (40, 2048, 9000)])
def test_digits_of_fp32_logits(n, f, c):
    s, _ = make(n, f, c, "f32", bias=False)
    got = top(s, 64)
    x, w = s["x"].double(), s["w"].double()
    z = x @ w
    want = z.gather(1, got["ids"].long())
    assert close(got["values"], want) <= most_off(f)
    assert close(got["lse"], torch.logsumexp(z, 1)) <= most_off(f, 3.0)
    if f <= 300:                                          # or the bound would let it pass
        lost = (two_parts(x) @ two_parts(w)).gather(1, got["ids"].long())
        assert close(lost, want) > 2 * most_off(f)


@pytest.mark.parametrize("n, f, c", PATHS)
def test_digits_of_fp32_gradients(n, f, c):
    """The gradient at the logits is off by the logits' error, the exponent's and the exponential's rounding: eight units at most, most of them of small probabilities."""
    s, _ = make(n, f, c, "f32", bias=False, labelled=1.0)
    got = forward(s)
    grads = backward(s, got["lse"], "f32", scale=1.0)
    x, w = s["x"].double(), s["w"].double()
    g = torch.exp(x @ w - got["lse"].double()[:, None])
    g.scatter_add_(1, s["labels"].long()[:, None], torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda"))
    for name, a, b, k in (("gx", g, w.t(), c), ("gw", x.t(), g, n)):
        want = a @ b
        assert close(grads[name], want) <= most_off(k, 8.0), name
        if k < 10_000:
            assert close(two_parts(a) @ two_parts(b), want) > most_off(k, 8.0), name
    assert close(grads["gbias"], g.sum(0)) <= most_off(n, 8.0)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n, f, c", [(1, 2048, 4001), (1, 1500, 16_000), (3, 1100, 20_001), (8, 512, 40_000), (8, 600, 40_003), (5, 1600, 300)])
def test_top_logits_of_few_rows_in_split_sums(n, f, c, dtype):
    s = exact_layer(n, f, c, dtype)
    got = top(s, 33)
    z = s["x"].double() @ s["w"].double() + s["bias"].double()
    ids, values = R.top(z, 33)
    assert torch.equal(got["ids"].long(), ids) and torch.equal(got["values"].double(), values)
    lse, off = R.log_sum_exp(z, torch.zeros_like(z))
    check(got["lse"], (lse.cpu(), off.cpu()), "lse")
