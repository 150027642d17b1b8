"""A residual model with classes by the thousand: its training steps without logits against the ones that keep them, a teacher's top logits, and its student."""
import pytest
import torch

from paper_2106_05609_amd import binding as B
from tests import classes_reference as R
from tests.test_gpu_residual_model import _setting
from tests.util import max_rel_err, to_np

pytestmark = pytest.mark.gpu
CLASSES = 1500


def setting(dtype, seed=0):
    return _setting(1, 0.1, dtype, 128, 64, CLASSES, 3, B.NORM_RMS, True, True, seed)


def labels_of(nb):
    gen = torch.Generator().manual_seed(3)
    labels = torch.randint(0, CLASSES, (nb,), generator=gen).int()
    labels[torch.rand(nb, generator=gen) < 0.6] = -1
    return labels.cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_without_logits(dtype):
    """The loss and every gradient as with them: of fp32 sums in another order; of bf16 the gradient at the logits is rounded once on either path, there times
    the scale, and the logits themselves with them only, by half a step of up to 4 (2^-7 of a probability)."""
    got = []
    for keep in (True, False):
        residual, model, g, sg, bg, x, hist = setting(dtype)
        opt = residual.AdamW(model.tensors(), 1e-3, max_norm=1.0)
        loss, n, y, grads = residual.residual_train_step(model, bg, x, hist, labels_of(sg.nb), opt, keep_logits=keep)
        assert (y is None) == (not keep) and n == int((labels_of(sg.nb) >= 0).sum())
        got.append((loss.item(), [v.clone() for v in grads], hist))
    (la, ga, ha), (lb, gb, hb) = got
    tol = 3e-5 if dtype == torch.float32 else 3e-2
    assert abs(la - lb) <= (1e-6 if dtype == torch.float32 else 2 ** -7) * abs(la)
    for k, (a, b) in enumerate(zip(ga, gb)):
        assert a.dtype == b.dtype == torch.float32 and max_rel_err(to_np(b), to_np(a.double())) <= tol, k
    assert all(torch.equal(a, b) for a, b in zip(ha, hb))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_teacher_teaches(dtype):
    """Its top logits as they come out, a student's step from them and labels, and the gradients against ones that go through all logits in 64 bits."""
    residual, teacher, g, sg, bg, x, hist = setting(dtype, seed=1)
    before = [h.clone() for h in hist]
    ids, values, lse = residual.residual_top(teacher, bg, x, hist, 20)
    assert all(torch.equal(a, b) for a, b in zip(hist, before))
    u = residual.residual_forward_batch(teacher, bg, x, hist, do_push=False, logits=False)
    z = u.double().cpu() @ teacher.w_out.double().cpu()
    assert (values.double().cpu() - z.topk(20, 1).values).abs().max() <= 64 * 256 * R.U32 and (lse.double().cpu() - torch.logsumexp(z, 1)).abs().max() <= 64 * 256 * R.U32
    _, student, _, _, _, _, hist = setting(dtype, seed=2)
    labels, t, weight = labels_of(sg.nb), 2.0, 0.3
    start = [h.clone() for h in hist]
    opt = residual.AdamW(student.tensors(), 1e-3)
    weights = [w.clone() for w in student.tensors()]
    loss, grads = residual.residual_distill_step(student, bg, x, hist, ids, values, opt, t, labels, weight)
    assert opt.steps.item() == 1 and not any(torch.equal(a, b) for a, b in zip(weights, student.tensors()))
    for w, old in zip(student.tensors(), weights):
        w.copy_(old)
    seen = {}

    def head(u, w, gu, gw):
        x64, w64 = u.double().cpu(), w.double().cpu()
        want = R.distill(x64, w64, None, ids.cpu(), values.cpu(), t, labels.cpu(), weight)
        gz, _ = R.grad_at_logits(x64, w64, None, want["lse"][0], labels.cpu(), None, ids.cpu(), values.cpu(), t, weight)
        gz /= sg.nb
        gu.copy_((gz @ w64.t()).to(gu))
        gw.copy_((x64.t() @ gz).to(gw))
        seen["loss"] = want["loss"][0].sum().item()
    _, want, _ = residual.residual_train_batch(student, bg, x, start, head=head)
    assert abs(loss.item() - seen["loss"]) <= (1e-6 if dtype == torch.float32 else 1e-5) * abs(seen["loss"])
    tol = 3e-5 if dtype == torch.float32 else 3e-2
    for k, (a, b) in enumerate(zip(grads, want)):
        assert max_rel_err(to_np(a), to_np(b.double())) <= tol, k


def test_a_step_without_logits_as_a_graph():
    """Captured once, replayed with eager work in between: as without."""
    runs = []
    for graph in (False, True):
        residual, model, g, sg, bg, x, hist = setting(torch.float32)
        opt = residual.AdamW(model.tensors(), 1e-2, bits=8, max_norm=0.5)
        labels = labels_of(sg.nb)
        one = lambda: residual.residual_train_step(model, bg, x, hist, labels, opt, n_labelled=100, keep_logits=False)[0]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            one()
        torch.cuda.synchronize()
        if graph:
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                loss = one()
            losses = []
            for _ in range(4):
                captured.replay()
                losses.append(float(loss))
                torch.randn(1000, device="cuda").sum().item()
        else:
            losses = [float(one()) for _ in range(4)]
        runs.append((losses, model.tensors() + hist))
    assert runs[0][0] == runs[1][0] and all(torch.equal(a, b) for a, b in zip(runs[0][1], runs[1][1]))


def test_one_or_the_other():
    residual, model, g, sg, bg, x, hist = setting(torch.float32)
    for kw in ({}, dict(grad_out=torch.zeros(sg.nb, CLASSES, device="cuda"), head=lambda *a: None)):
        with pytest.raises(ValueError, match="either grad_out or head"):
            residual.residual_train_batch(model, bg, x, hist, **kw)
