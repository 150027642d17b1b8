"""A deep residual graph convolutional model for mini-batches with histories, and its training by AdamW.

As in executor.py nothing is computed here: buffers are torch allocations and every step is a gas_* call.  For a batch B with halo
V_b \\ B and widths F throughout:

    h_0 = x W_in                                         for every node of V_b
    u_l = N_pre(h_{l-1}) * q_l + q_bias_l                the layer's input; the next layers' histories hold u of the other batches
    a_l = relu((aggregation of u_l) W_l),  t_l = u_l V_l
    h_l = h_{l-1} + s_l * sigmoid(t_l) * (N_post(a_l) * p_l + p_bias_l)
    y   = (N_pre(h_L) * q_{L+1} + q_bias_{L+1}) W_out

What is between two layers, norm after the block, gate, residual scale, stream, norm before the next block and the Push of its
rows, is one call (gas_residual_norm).  Histories are constants in the backward pass (paper, Section 2).
"""
import torch

from . import binding as B
from .executor import BatchGraph, _pushes, _WeightGrads


class ResidualModel:
    """w_in [F0, F], layers: dicts of w [F, F], v [F, F] (None: no gate), p, p_bias, s (float32 [F], None: 1, 0, 1), w_out [F, C], and
    pre: L + 1 pairs (q, q_bias) of the norms before the blocks and before w_out."""

    def __init__(self, w_in, layers, pre, w_out, norm=B.NORM_RMS, eps=1e-5):
        if len(layers) == 0 or len(pre) != len(layers) + 1:
            raise ValueError(f"ResidualModel: {len(pre)} norms before {len(layers)} blocks and the output")
        self.w_in, self.layers, self.pre, self.w_out, self.norm, self.eps = w_in, layers, pre, w_out, norm, eps

    @property
    def n_layers(self):
        return len(self.layers)

    def tensors(self):
        """Every tensor that is learned, in the order of the gradients."""
        ts = [self.w_in, self.w_out]
        for layer in self.layers:
            ts += [layer["w"], layer["v"], layer["p"], layer["p_bias"], layer["s"]]
        for q in self.pre:
            ts += q
        return [t for t in ts if t is not None]


def residual_forward_batch(model: ResidualModel, bg: BatchGraph, x_feat, histories, do_push=True, keep=None):
    """All layers for one mini-batch in the order of Algorithm 1: y [nb, C].  histories[l - 1]: table [N, F] of u_{l+1}, l = 1 .. L - 1.  keep: a
    dict that receives what the backward pass reads."""
    dev, dt, nb, nv, f = x_feat.device, x_feat.dtype, bg.nb, bg.nv, model.w_in.shape[1]
    new = lambda rows, cols=f: torch.empty((rows, cols), dtype=dt, device=dev)
    stats_of = lambda rows: None if keep is None else torch.empty((rows, 4), dtype=torch.float32, device=dev)
    ids, L, norm = bg.n_id[:nb], model.n_layers, dict(pre=model.norm, eps=model.eps)
    x0, h0, x = new(nv, x_feat.shape[1]), new(nv), new(nv)
    B.gas_pull(x_feat, bg.n_id, x0)
    B.gas_linear(x0, model.w_in, h0)
    stats0 = stats_of(nv)
    q, q_bias = model.pre[0]
    B.gas_residual_norm(h0, u=x, q=q, q_bias=q_bias, stats=stats0, **norm)
    h, saved = h0[:nb], []
    for l in range(1, L + 1):
        layer, (q, q_bias) = model.layers[l - 1], model.pre[l]
        z, a, t = new(nb), new(nb), None if layer["v"] is None else new(nb)
        if l == 1:
            B.gas_spmm(bg.plan, bg.rowptr, bg.col, bg.val, x, z)
        else:                                 # halo rows in place, from the history of the layer below
            B.gas_spmm_hist(bg.plan, bg.rowptr, bg.src, bg.val, x, histories[l - 2], z)
        B.gas_linear(z, layer["w"], a, relu=True)
        if t is not None:
            B.gas_linear(x[:nb], layer["v"], t)
        h_next, u, stats = new(nb) if l < L or keep is not None else None, new(nb), stats_of(nb)
        push = l < L and _pushes(do_push, histories[l - 1])
        B.gas_residual_norm(h, h=h_next, u=u, a=a, t=t, post=model.norm, p=layer["p"], p_bias=layer["p_bias"], s=layer["s"], q=q, q_bias=q_bias,
                            stats=stats, idx=ids if push else None, hist=histories[l - 1] if push else None, **norm)
        if l < L and do_push and not push:
            B.gas_push(u, ids, histories[l - 1])
        saved.append((x[:nb], z, a, t, h_next, stats))
        x, h = u, h_next
    y = new(nb, model.w_out.shape[1])
    B.gas_linear(x, model.w_out, y)
    if keep is not None:
        keep.update(x0=x0, h0=h0, stats0=stats0, layers=saved, u=x)
    return y


def residual_train_batch(model: ResidualModel, bg: BatchGraph, x_feat, histories, grad_out, do_push=True):
    """residual_forward_batch and its backward pass; bg needs the CSC copy.  grad_out: dLoss/dy [nb, C] or a function of y.  Returns (y, grads,
    kept) with the gradients, float32, of model.tensors() in their order."""
    kept = {}
    y = residual_forward_batch(model, bg, x_feat, histories, do_push, kept)
    dev, dt, nb, nv, f, L = x_feat.device, x_feat.dtype, bg.nb, bg.nv, model.w_in.shape[1], model.n_layers
    new = lambda rows: torch.empty((rows, f), dtype=dt, device=dev)
    like = lambda v: None if v is None else torch.empty_like(v)
    wg = _WeightGrads()
    gy = grad_out(y) if callable(grad_out) else grad_out
    g_out = wg.add(kept["u"], gy)
    gu, gh = new(nb), None
    B.gas_linear_bwd_input(gy, model.w_out, gu)
    room = torch.empty(max(1, B.gas_residual_norm_bwd_workspace(nv, f, dt)), dtype=torch.uint8, device=dev)
    g_layers, g_pre = [None] * L, [None] * (L + 1)
    for l in range(L, 0, -1):
        layer, (q, q_bias) = model.layers[l - 1], model.pre[l]
        u, z, a, t, h, stats = kept["layers"][l - 1]
        # the first layer's stream is the in-batch part of h_0, whose other rows no stream leaves
        gx = new(nb) if l > 1 else torch.zeros((nv, f), dtype=dt, device=dev)
        ga, gt = new(nb), like(t)
        g = dict(p=like(layer["p"]), p_bias=like(layer["p_bias"]), s=like(layer["s"]))
        g_pre[l] = (like(q), like(q_bias))
        B.gas_residual_norm_bwd(gh, gu, h, stats, gx=gx[:nb], ga=ga, gt=gt, a=a, t=t, post=model.norm, p=layer["p"], p_bias=layer["p_bias"],
                                s=layer["s"], pre=model.norm, q=q, gp=g["p"], gp_bias=g["p_bias"], gs=g["s"], gq=g_pre[l][0], gq_bias=g_pre[l][1],
                                workspace=room)
        B.gas_relu_bwd(ga, a, ga)
        g["w"], g["v"] = wg.add(z, ga), None if t is None else wg.add(u, gt)
        g_layers[l - 1] = g
        gz = new(nb)
        B.gas_linear_bwd_input(ga, layer["w"], gz)
        gu = new(nb if l > 1 else nv)
        B.gas_spmm_t(bg.plan_t if l > 1 else bg.plan_t_all, bg.colptr, bg.row, bg.val_t, gz, gu)
        if t is not None:                     # the gate reads the in-batch rows of u too
            part = new(nb)
            if l > 1:
                B.gas_linear_bwd_input_add(gt, layer["v"], part, add=gu)
                gu = part
            else:
                B.gas_linear_bwd_input(gt, layer["v"], part)
                B.gas_axpy(gu[:nb], part, gu[:nb], 1.0)
        gh = gx
    g_pre[0] = tuple(like(v) for v in model.pre[0])
    g0 = new(nv)
    B.gas_residual_norm_bwd(gh, gu, kept["h0"], kept["stats0"], gx=g0, pre=model.norm, q=model.pre[0][0], gq=g_pre[0][0], gq_bias=g_pre[0][1],
                            workspace=room)
    g_in = wg.add(kept["x0"], g0)
    wg.done()
    grads = [g_in, g_out]
    for g in g_layers:
        grads += [g["w"], g["v"], g["p"], g["p_bias"], g["s"]]
    for g in g_pre:
        grads += g
    return y, [g for g in grads if g is not None], kept


class AdamW:
    """The AdamW step of a list of tensors (float32 or bfloat16) with gradients in float32, clipped by their global norm.  bits: of the states; with 8,
    tensors of fewer than SMALL elements keep 32, which costs little and keeps gains and biases exact.  bfloat16 tensors are
    updated through float32 masters, so they must not share memory.  Tensors with one dimension (gains, biases) are not decayed.  A step whose gradients hold an infinity or a NaN
    changes nothing, the number of steps included.  The number is kept on the device, so a captured step() counts on."""
    SMALL = 4096

    def __init__(self, tensors, lr, bits=32, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_norm=float("inf")):
        if bits not in (8, 32):
            raise ValueError(f"AdamW: states of {bits} bits")
        self.tensors, self.lr, self.max_norm = list(tensors), lr, max_norm
        if not self.tensors:
            raise ValueError("AdamW: no tensors")
        spans = sorted((t.data_ptr(), t.data_ptr() + 2 * t.numel()) for t in self.tensors if t.dtype == torch.bfloat16 and t.numel())
        if any(one[1] > next_[0] for one, next_ in zip(spans, spans[1:])):
            raise ValueError("AdamW: bfloat16 tensors that share memory, each with a master of its own: only the last one's gradient would count")
        self.hyper = dict(beta1=beta1, beta2=beta2, eps=eps)
        dev = self.tensors[0].device
        self.steps, self.sq_norm = torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros(1, device=dev)
        self.groups = []
        for eight in (True, False):
            picked = [i for i, t in enumerate(self.tensors) if (bits == 8 and t.numel() >= self.SMALL) == eight]
            if not picked:
                continue
            ws = [self.tensors[i] for i in picked]
            sizes = [w.numel() for w in ws]
            n = B.gas_adamw_elements(sizes)
            new = lambda dt: torch.zeros(n, dtype=dt, device=dev)
            g = dict(picked=picked, ws=ws, decay=[weight_decay if w.dim() > 1 else 0.0 for w in ws],
                     m=new(torch.int8 if eight else torch.float32), v=new(torch.uint8 if eight else torch.float32),
                     scales=torch.zeros((n // 256, 2), device=dev) if eight else None, master=None)
            if any(w.dtype == torch.bfloat16 for w in ws):
                g["master"], at = new(torch.float32), 0
                for w in ws:
                    g["master"][at:at + w.numel()] = w.reshape(-1).float()
                    at += -(-w.numel() // 256) * 256
            self.groups.append(g)

    def step(self, grads):
        """One update of the tensors, in place."""
        if len(grads) != len(self.tensors):
            raise ValueError(f"AdamW: {len(grads)} gradients of {len(self.tensors)} tensors")
        B.gas_sq_norms(grads, self.sq_norm, steps=self.steps)
        for g in self.groups:
            B.gas_adamw_steps(g["ws"], [grads[i] for i in g["picked"]], g["m"], g["v"], self.lr, weight_decay=g["decay"], scales=g["scales"],
                              master=g["master"], steps=self.steps, sq_norm=self.sq_norm, max_norm=self.max_norm, **self.hyper)

    def states(self):
        """(m, v) of every tensor in float32, as the state holds them or, of 8 bits, what it stands for."""
        out = [None] * len(self.tensors)
        for g in self.groups:
            m, v = g["m"], g["v"]
            if g["scales"] is not None:
                m, v = (torch.empty(g["m"].numel(), device=g["m"].device) for _ in range(2))
                B.gas_adamw_unpack(g["m"], g["v"], g["scales"], m, v)
            at = 0
            for i, w in zip(g["picked"], g["ws"]):
                out[i] = (m[at:at + w.numel()].view(w.shape), v[at:at + w.numel()].view(w.shape))
                at += -(-w.numel() // 256) * 256
        return out


def residual_train_step(model: ResidualModel, bg: BatchGraph, x_feat, histories, labels_batch, optimizer: AdamW, n_labelled=None, do_push=True):
    """One optimisation step on one mini-batch: forward with Push, softmax cross-entropy averaged over the labelled in-batch nodes
    (labels_batch int32 [nb], < 0 = unlabelled; n_labelled: their count if the caller knows it), backward, AdamW.  Returns (loss_sum as a 1-element device
    tensor, n_labelled, y, grads)."""
    if n_labelled is None:
        n_labelled = int((labels_batch >= 0).sum().item())
    dev = x_feat.device
    loss_rows, loss_sum = torch.empty(bg.nb, dtype=torch.float32, device=dev), torch.empty(1, dtype=torch.float32, device=dev)

    def loss_grad(y):
        g = torch.empty_like(y)
        B.gas_softmax_xent(y, labels_batch, g, loss_rows, loss_sum, scale=1.0 / max(1, n_labelled))
        return g
    y, grads, _ = residual_train_batch(model, bg, x_feat, histories, loss_grad, do_push)
    optimizer.step(grads)
    return loss_sum, n_labelled, y, grads
