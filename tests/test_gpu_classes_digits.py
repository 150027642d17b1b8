"""Digits of the products of an output layer over many classes on every path that its sizes choose, and ties between classes that different launches form."""
import math

import pytest
import torch

import paper_2106_05609_amd as gas
from tests import classes_reference as R
from tests.test_gpu_classes import DT, backward, close, forward, make, top

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
