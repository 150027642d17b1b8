"""What the calls of an output layer over many classes refuse, before anything is launched (no GPU here)."""
import pytest
import torch

import paper_2106_05609_amd as gas
from paper_2106_05609_amd import binding

N, F, C, K = 6, 16, 40, 3


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)


def args(dt=torch.float32):
    return dict(x=torch.zeros(N, F, dtype=dt), w=torch.zeros(F, C, dtype=dt), labels=torch.zeros(N, dtype=torch.int32), loss=torch.zeros(N),
                lse=torch.zeros(N), lse2=torch.zeros(N, 2), ids=torch.zeros(N, K, dtype=torch.int32), values=torch.zeros(N, K))


def xent(a, **kw):
    gas.gas_linear_xent(a["x"], a["w"], a["labels"], a["loss"], a["lse"], **kw)


def xent_bwd(a, **kw):
    kw = dict(dict(gx=torch.zeros_like(a["x"])), **kw)
    gas.gas_linear_xent_bwd(a["x"], a["w"], a["labels"], a["lse"], **kw)


def distill(a, **kw):
    gas.gas_linear_distill(a["x"], a["w"], a["ids"], a["values"], a["loss"], a["lse2"], **kw)


def distill_bwd(a, **kw):
    kw = dict(dict(gx=torch.zeros_like(a["x"])), **kw)
    gas.gas_linear_distill_bwd(a["x"], a["w"], a["ids"], a["values"], a["lse2"], **kw)


def top(a, **kw):
    gas.gas_linear_top(a["x"], a["w"], a["ids"], a["values"], **kw)


EVERY = [xent, xent_bwd, distill, distill_bwd, top]


@pytest.mark.parametrize("call", EVERY)
def test_shapes_and_dtypes_of_the_layer(call):
    for key, bad in (("x", torch.zeros(N, F + 1)), ("w", torch.zeros(F, C, dtype=torch.bfloat16)), ("x", torch.zeros(N, F, dtype=torch.float16)),
                     ("x", torch.zeros(N, F, dtype=torch.float64)), ("x", torch.zeros(F, N).t()), ("w", torch.zeros(C, F).t())):
        with pytest.raises((ValueError, TypeError)):
            call(dict(args(), **{key: bad}))
    for bias in (torch.zeros(C + 1), torch.zeros(C, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="do not match"):
            call(args(), bias=bias)


@pytest.mark.parametrize("call, key, bad", [
    (xent, "labels", torch.zeros(N + 1, dtype=torch.int32)), (xent, "labels", torch.zeros(N, dtype=torch.int64)), (xent, "loss", torch.zeros(N - 1)),
    (xent, "lse", torch.zeros(N, dtype=torch.float64)), (xent_bwd, "lse", torch.zeros(N, 2)), (xent_bwd, "labels", torch.zeros(2 * N, dtype=torch.int32)[::2]),
    (distill, "ids", torch.zeros(N, K, dtype=torch.int64)), (distill, "ids", torch.zeros(N, K + 1, dtype=torch.int32)),
    (distill, "values", torch.zeros(N, K, dtype=torch.bfloat16)), (distill, "values", torch.zeros(N + 1, K)), (distill, "lse2", torch.zeros(2, N)),
    (distill_bwd, "lse2", torch.zeros(N)), (top, "ids", torch.zeros(N, K, dtype=torch.int64)), (top, "values", torch.zeros(N, K + 1))])
def test_shapes_and_dtypes_of_the_rest(call, key, bad):
    with pytest.raises((ValueError, TypeError)):
        call(dict(args(), **{key: bad}))


@pytest.mark.parametrize("call, kw", [
    (xent_bwd, dict(gx=None)), (xent_bwd, dict(gw=torch.zeros(F, C, dtype=torch.bfloat16))), (distill, dict(temperature=0.0)),
    (distill, dict(temperature=-1.0)), (distill, dict(temperature=float("inf"))), (distill, dict(temperature=float("nan"))),
    (distill, dict(label_weight=1.5)), (distill_bwd, dict(label_weight=-0.1)), (distill_bwd, dict(label_weight=float("nan")))])
def test_values_that_no_call_takes(call, kw):
    with pytest.raises(gas.GasError) as e:
        call(args(), **kw)
    assert e.value.status in (-1, -2)


@pytest.mark.parametrize("call, kw", [(xent_bwd, dict(gx=torch.zeros(N, F + 1))), (xent_bwd, dict(gw=torch.zeros(C, F))), (xent_bwd, dict(gbias=torch.zeros(F))),
                                      (xent_bwd, dict(gbias=torch.zeros(C, dtype=torch.bfloat16))), (xent_bwd, dict(row_scale=torch.zeros(N + 1))),
                                      (xent, dict(loss_sum=torch.zeros(1, dtype=torch.float64)))])
def test_shapes_of_optional_arguments(call, kw):
    with pytest.raises((ValueError, TypeError)):
        call(args(), **kw)


def test_entries_of_a_row():
    many = 257
    with pytest.raises(gas.GasError, match="1 to 256 entries"):
        distill(dict(args(), ids=torch.zeros(N, many, dtype=torch.int32), values=torch.zeros(N, many)))
    for k in (0, 129, C + 1):
        with pytest.raises(gas.GasError, match="are taken"):
            top(dict(args(), ids=torch.zeros(N, k, dtype=torch.int32), values=torch.zeros(N, k)))


@pytest.mark.parametrize("call", EVERY)
def test_a_workspace_that_is_too_small(call):
    with pytest.raises(gas.GasError, match="are needed"):
        call(args(), workspace=torch.zeros(64, dtype=torch.uint8))


def room(call):
    w = {xent: gas.gas_linear_xent_workspace, xent_bwd: gas.gas_linear_xent_bwd_workspace}
    if call in w:
        return w[call](N, F, C, torch.float32)
    return {distill: gas.gas_linear_distill_workspace, distill_bwd: gas.gas_linear_distill_bwd_workspace, top: gas.gas_linear_top_workspace}[call](
        N, F, C, torch.float32, K)


@pytest.mark.parametrize("call", EVERY)
def test_outputs_that_overlap(call):
    """Refused whatever overlaps: two outputs, or an output and an input or the workspace."""
    a, cases = args(), []
    flat = torch.zeros(4096)
    if call in (xent, distill):
        lse = "lse" if call is xent else "lse2"
        cases = [(dict(a, loss=flat[:N], **{lse: flat[1:1 + a[lse].numel()].view(a[lse].shape)}), {}), (dict(a, loss=a["x"].view(-1)[:N]), {}),
                 (a, dict(loss_sum=a["loss"][2:3])), (dict(a, loss=a["w"].view(-1)[7:7 + N]), {})]
    elif call is top:
        cases = [(dict(a, values=a["x"][:, 2:2 + K]), {}), (dict(a, values=flat[:N * K].view(N, K), ids=flat[:N * K].view(torch.int32).view(N, K)), {}),
                 (a, dict(lse=a["values"].view(-1)[3:3 + N]))]
    else:
        cases = [(a, dict(gx=a["x"])), (a, dict(gw=a["w"])), (a, dict(gbias=a["w"][3])), (a, dict(gx=flat[:N * F].view(N, F), gw=flat[F:F + F * C].view(F, C)))]
    work = torch.zeros(room(call) + 4096, dtype=torch.uint8)
    first = work.view(torch.float32)
    if call in (xent, distill):
        cases.append((dict(a, loss=first[8:8 + N]), dict(workspace=work)))
    elif call is top:
        cases.append((dict(a, values=first[8:8 + N * K].view(N, K)), dict(workspace=work)))
    else:
        cases.append((a, dict(gx=first[8:8 + N * F].view(N, F), workspace=work)))
    for b, kw in cases:
        with pytest.raises(gas.GasError, match="overlap"):
            call(b, **kw)


@pytest.mark.parametrize("call", EVERY)
def test_tensors_on_another_device(call):
    a = args()
    with pytest.raises((ValueError, TypeError, RuntimeError)):
        call(dict(a, w=torch.zeros(F, C, device="meta")))


def test_workspaces_are_known_for_what_calls_take():
    assert gas.gas_linear_xent_workspace(0, F, C, torch.float32) == 0
    for n, f, c in ((-1, F, C), (N, 0, C), (N, F, 0), (N, 1 << 17, C), (N, F, (1 << 22) + 1), (1 << 29, F, C)):
        assert gas.gas_linear_xent_workspace(n, f, c, torch.float32) == -1
        assert gas.gas_linear_xent_bwd_workspace(n, f, c, torch.bfloat16) == -1
    for k in (0, 257):
        assert gas.gas_linear_distill_workspace(N, F, C, torch.float32, k) == -1
    for k in (0, 129, C + 1):
        assert gas.gas_linear_top_workspace(N, F, C, torch.float32, k) == -1
    # a launch's threads are counted in 32 bits
    assert gas.gas_linear_xent_workspace(2 ** 25, 1, 2, torch.float32) > 0 > gas.gas_linear_xent_workspace(2 ** 25 + 1, 1, 2, torch.float32)
    assert gas.gas_linear_top_workspace(2 ** 23, 1, 2, torch.float32, 1) > 0 > gas.gas_linear_top_workspace(2 ** 23 + 1, 1, 2, torch.float32, 1)
    # the logits are not in it: less than they take, from a few thousand classes and rows on
    for dt, eb in ((torch.float32, 4), (torch.bfloat16, 2)):
        n, c = 100_000, 500_000
        assert gas.gas_linear_xent_workspace(n, 256, c, dt) < 0.05 * n * c * eb
        assert gas.gas_linear_xent_bwd_workspace(n, 256, c, dt) < 0.1 * n * c * eb
        assert gas.gas_linear_distill_bwd_workspace(n, 256, c, dt, 64) < 0.1 * n * c * eb
        assert gas.gas_linear_top_workspace(n, 256, c, dt, 64) < 0.1 * n * c * eb
