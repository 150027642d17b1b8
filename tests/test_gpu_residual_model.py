"""The residual model of paper_2106_05609_amd/residual.py on mini-batches with histories: a pass, its pushes and all gradients against the
same model in 64 bits with automatic differentiation, training by AdamW, and a training step as a HIP graph."""
import pytest
import torch

from gas_inputs import batches, configs, rng
from paper_2106_05609_amd import binding as B
from tests import residual_reference as R
from tests.util import max_rel_err, node_rel_err, to_np

pytestmark = pytest.mark.gpu
# as for the other operators' models: forward, and gradients behind up to some ten rounded tensors a layer
TOL = {torch.float32: (1e-5, 3e-5), torch.bfloat16: (2e-2, 3e-2)}


def _setting(cfg_id, scale, dtype, f0, f, classes, L, norm, gated, bias, seed=0):
    from paper_2106_05609_amd import executor, residual
    cfg = configs.config(cfg_id, scale)
    g = configs.build_graph(cfg)
    bl = batches.split(g, cfg.blocks_per_batch, cfg.seed)
    d = lambda t: t.to("cuda")
    gen = torch.Generator().manual_seed(seed)
    vec = lambda around: d(around + 0.1 * torch.randn(f, generator=gen))
    mat = lambda k, a, b: d(rng.glorot_uniform(cfg.seed, 1900 + k, a, b, dtype=dtype))
    layers = [dict(w=mat(2 * l, f, f), v=mat(2 * l + 1, f, f) if gated else None, p=vec(1.0), p_bias=vec(0.0) if bias else None, s=vec(0.5)) for l in range(L)]
    pre = [(vec(1.0), vec(0.0) if bias else None) for _ in range(L + 1)]
    model = residual.ResidualModel(mat(500, f0, f), layers, pre, mat(501, f, classes), norm)
    sg = batches.batch_subgraph(g, bl[0], True)
    bg = executor.BatchGraph(sg.nb, d(sg.n_id), d(sg.rowptr), d(sg.col), d(g.deg), d(sg.colptr), d(sg.row), max_F=max(f, f0))
    x = d(rng.normal_matrix(cfg.seed, 1950, g.n, f0, dtype=dtype))
    hist = [d(rng.normal_matrix(cfg.seed, 1960 + l, g.n, f, dtype=dtype)) for l in range(L - 1)]
    return residual, model, g, sg, bg, x, hist


def _reference(model, sg, bg, x, hist, masks, gout):
    """(y, what is pushed, gradients of model.tensors()) in 64 bits; masks: which units of a_l pass."""
    w64 = lambda t: None if t is None else t.double().cpu()
    leaves = [w64(t).requires_grad_() for t in model.tensors()]
    it = iter(leaves)
    w_in, w_out = next(it), next(it)
    layers = [{k: None if layer[k] is None else next(it) for k in ("w", "v", "p", "p_bias", "s")} for layer in model.layers]
    pre = [tuple(None if v is None else next(it) for v in q) for q in model.pre]
    nb, n_id = sg.nb, sg.n_id.long().cpu()
    rows = torch.repeat_interleave(torch.arange(nb), (sg.rowptr[1:] - sg.rowptr[:-1]).long().cpu())
    val = bg.val.double().cpu()
    a_hat = torch.sparse_coo_tensor(torch.stack([rows, sg.col.long().cpu()]), val, (nb, sg.nv)).to_dense()
    norm = lambda h, q: R.forward(h, None, None, 0, None, None, None, 1.0, model.norm, *q, model.eps)[1]
    h0 = w64(x)[n_id] @ w_in
    u_all, h, pushed = norm(h0, pre[0]), h0[:nb], []
    for l, layer in enumerate(layers):
        a = (a_hat @ u_all @ layer["w"]) * masks[l]
        t = None if layer["v"] is None else u_all[:nb] @ layer["v"]
        h, u, _ = R.forward(h, a, t, model.norm, layer["p"], layer["p_bias"], layer["s"], 1.0, model.norm, *pre[l + 1], model.eps)
        if l + 1 < len(layers):
            pushed.append(u)
            u_all = torch.cat([u, w64(hist[l])[n_id[nb:]]])
    y = u @ w_out
    (y * w64(gout)).sum().backward()
    return y.detach(), [p.detach() for p in pushed], [t.grad for t in leaves]


@pytest.mark.parametrize("cfg_id,scale,dtype,f0,f,classes,L,norm,gated,bias", [
    (1, 0.1, torch.float32, 100, 64, 47, 3, B.NORM_LAYER, True, True),
    (1, 0.1, torch.float32, 128, 256, 40, 2, B.NORM_RMS, True, False),
    (1, 0.1, torch.float32, 24, 47, 7, 4, B.NORM_RMS, False, False),
    (2, 0.01, torch.float32, 100, 100, 47, 1, B.NORM_LAYER, True, True),
    (1, 0.1, torch.bfloat16, 128, 64, 16, 2, B.NORM_RMS, True, True),
    (1, 0.1, torch.bfloat16, 128, 256, 16, 3, B.NORM_LAYER, False, True)])
def test_pass_and_gradients(cfg_id, scale, dtype, f0, f, classes, L, norm, gated, bias):
    residual, model, g, sg, bg, x, hist = _setting(cfg_id, scale, dtype, f0, f, classes, L, norm, gated, bias)
    gout = rng.normal_matrix(7, 1970, sg.nb, classes, dtype=dtype).to("cuda")
    before = [t.clone() for t in hist]
    y, grads, kept = residual.residual_train_batch(model, bg, x, hist, gout)
    masks = [(layer[2] > 0).double().cpu() for layer in kept["layers"]]
    want_y, pushed, want = _reference(model, sg, bg, x, before, masks, gout)
    fwd, bwd = TOL[dtype]
    assert node_rel_err(to_np(y), want_y.numpy()) <= fwd
    ids = sg.n_id[:sg.nb].long().cuda()
    for table, old, u in zip(hist, before, pushed):
        assert node_rel_err(to_np(table[ids]), u.numpy()) <= fwd
        rest = torch.ones(g.n, dtype=torch.bool, device="cuda")
        rest[ids] = False
        assert torch.equal(table[rest], old[rest])
    assert len(grads) == len(want) == len(model.tensors())
    for k, (got, w) in enumerate(zip(grads, want)):
        assert got.shape == w.shape and got.dtype == torch.float32
        assert max_rel_err(to_np(got), w.numpy()) <= bwd, k
    # inference gives the same rows, and a second pass the same bits
    again = [t.clone() for t in before]
    assert torch.equal(residual.residual_forward_batch(model, bg, x, again), y) and all(torch.equal(a, b) for a, b in zip(again, hist))
    y2, grads2, _ = residual.residual_train_batch(model, bg, x, before, gout, do_push=False)
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_training(dtype, bits):
    """Labels that a linear map of the smoothed features gives are learned: the loss falls to less than half in 40 steps."""
    residual, model, g, sg, bg, x, hist = _setting(1, 0.1, dtype, 128, 64, 8, 3, B.NORM_RMS, True, True)
    labels = (x.float()[sg.n_id[:sg.nb].long().cuda()] @ torch.randn(128, 8, generator=torch.Generator().manual_seed(5)).cuda()).argmax(1).int()
    labels[::7] = -1
    opt = residual.AdamW(model.tensors(), 3e-3, bits=bits, max_norm=1.0)
    losses = [float(residual.residual_train_step(model, bg, x, hist, labels, opt)[0]) for _ in range(40)]
    assert losses[-1] < 0.5 * losses[0] and opt.steps.item() == 40
    for (m, v), t in zip(opt.states(), model.tensors()):
        assert m.shape == v.shape == t.shape and torch.isfinite(m).all() and (v >= 0).all()
    if bits == 8:
        assert any(grp["scales"] is not None for grp in opt.groups) and any(grp["scales"] is None for grp in opt.groups)


def test_states_of_8_bits_train_as_those_of_32():
    """The same 60 steps: the sum of the last ten losses differs by a tenth at most."""
    got = []
    for bits in (32, 8):
        residual, model, g, sg, bg, x, hist = _setting(1, 0.1, torch.float32, 128, 64, 8, 3, B.NORM_RMS, True, True)
        labels = (x[sg.n_id[:sg.nb].long().cuda()] @ torch.randn(128, 8, generator=torch.Generator().manual_seed(5)).cuda()).argmax(1).int()
        opt = residual.AdamW(model.tensors(), 1e-3, bits=bits, max_norm=1.0)
        losses = [float(residual.residual_train_step(model, bg, x, hist, labels, opt)[0]) for _ in range(60)]
        got.append(sum(losses[-10:]))
    assert abs(got[1] - got[0]) <= 0.1 * got[0]


def test_a_training_step_as_a_graph():
    """Captured once, replayed with eager work in between: weights, states, histories and the step's number as without."""
    runs = []
    for graph in (False, True):
        residual, model, g, sg, bg, x, hist = _setting(1, 0.1, torch.float32, 128, 64, 8, 2, B.NORM_LAYER, True, True)
        labels = torch.randint(0, 8, (sg.nb,), generator=torch.Generator().manual_seed(2)).int().cuda()
        opt = residual.AdamW(model.tensors(), 1e-2, bits=8, max_norm=0.5)
        one = lambda: residual.residual_train_step(model, bg, x, hist, labels, opt, n_labelled=sg.nb)[0]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            one()                                            # builds what is built once
        torch.cuda.synchronize()
        losses = []
        if graph:
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                loss = one()
            for _ in range(5):
                captured.replay()
                losses.append(float(loss))
                torch.randn(1000, device="cuda").sum().item()
        else:
            losses = [float(one()) for _ in range(5)]
        runs.append((losses, model.tensors(), hist, opt))
    (la, ta, ha, oa), (lb, tb, hb, ob) = runs
    assert la == lb and oa.steps.item() == ob.steps.item() == 6
    assert all(torch.equal(a, b) for a, b in zip(ta + ha, tb + hb))
    for a, b in zip(oa.groups, ob.groups):
        assert torch.equal(a["m"], b["m"]) and torch.equal(a["v"], b["v"])


def test_an_infinity_is_skipped():
    residual, model, g, sg, bg, x, hist = _setting(1, 0.1, torch.float32, 128, 64, 8, 2, B.NORM_RMS, False, False)
    opt = residual.AdamW(model.tensors(), 1e-2)
    grads = [torch.ones(t.shape, device="cuda") for t in model.tensors()]
    before = [t.clone() for t in model.tensors()]
    grads[3].view(-1)[5] = float("inf")
    opt.step(grads)
    assert opt.steps.item() == 0 and all(torch.equal(a, b) for a, b in zip(before, model.tensors()))
    grads[3].view(-1)[5] = 1.0
    opt.step(grads)
    assert opt.steps.item() == 1 and not any(torch.equal(a, b) for a, b in zip(before, model.tensors()))


def test_refusals():
    from paper_2106_05609_amd import residual
    w = torch.zeros(8, 8, device="cuda")
    with pytest.raises(ValueError, match="1 norms before 1 blocks"):
        residual.ResidualModel(w, [dict(w=w, v=None, p=None, p_bias=None, s=None)], [(None, None)], w)
    with pytest.raises(ValueError, match="4 bits"):
        residual.AdamW([w], 0.1, bits=4)
    with pytest.raises(ValueError, match="2 gradients of 1"):
        residual.AdamW([w], 0.1).step([w, w])
