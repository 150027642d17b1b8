#!/usr/bin/env python3
"""Training of a deep residual model (paper_2106_05609_amd/residual.py) on the graph and batches of a benchmark configuration: for every
mini-batch forward with Push, softmax cross-entropy, backward, AdamW with the gradients clipped.  Every step is a C-ABI call.  One JSON line on
stdout: ms per epoch and step, and the loss of every epoch."""
import argparse
import json
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--config", type=int, default=1)
    p.add_argument("--scale", type=float, default=1.0)
    p.add_argument("--layers", type=int, default=8)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--norm", choices=["rms", "layer"], default="rms")
    p.add_argument("--no-gate", action="store_true")
    p.add_argument("--bits", type=int, choices=[8, 32], default=32, help="of the optimiser's states")
    p.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    p.add_argument("--epochs", type=int, default=3, help="timed epochs after one warm-up epoch")
    p.add_argument("--lr", type=float, default=1e-3)
    args = p.parse_args()
    if not torch.cuda.is_available():
        sys.exit("bench_residual.py: no GPU visible")
    import paper_2106_05609_amd as gas
    from paper_2106_05609_amd import executor, residual
    from gas_inputs import batches, configs, rng
    gas.lib()
    dev = torch.device("cuda:0")
    cfg = configs.config(args.config, args.scale)
    dt, f, L = torch.bfloat16 if args.dtype == "bf16" else torch.float32, args.width, args.layers
    g = configs.build_graph(cfg, device=dev)
    labels = configs.block_labels(g, 16, cfg.seed, unlabelled=0.5).to(dev)
    f0 = cfg.widths[0]
    mat = lambda k, a, b: rng.glorot_uniform(cfg.seed, 1900 + k, a, b, dev, dt)
    ones = lambda v=1.0: torch.full((f,), v, device=dev)
    layers = [dict(w=mat(2 * l, f, f), v=None if args.no_gate else mat(2 * l + 1, f, f), p=ones(), p_bias=None, s=ones(0.5)) for l in range(L)]
    model = residual.ResidualModel(mat(1000, f0, f), layers, [(ones(), None) for _ in range(L + 1)], mat(1001, f, 16),
                                   gas.NORM_RMS if args.norm == "rms" else gas.NORM_LAYER)
    x = rng.normal_matrix(cfg.seed, 1950, g.n, f0, dev, dt)
    hist = [torch.zeros((g.n, f), dtype=dt, device=dev) for _ in range(L - 1)]
    opt = residual.AdamW(model.tensors(), args.lr, bits=args.bits, max_norm=1.0)
    parts = []
    for b in batches.split(g, cfg.blocks_per_batch, cfg.seed):
        sg = batches.batch_subgraph(g, b, True).to(dev)
        bg = executor.BatchGraph(sg.nb, sg.n_id, sg.rowptr, sg.col, g.deg.to(dev), sg.colptr, sg.row, max_F=max(f, f0))
        mine = labels[sg.n_id[:sg.nb].long()].int().contiguous()
        parts.append((bg, mine, int((mine >= 0).sum().item())))
    torch.cuda.reset_peak_memory_stats()
    ms, losses = [], []
    for epoch in range(args.epochs + 1):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        sums = [residual.residual_train_step(model, bg, x, hist, mine, opt, n_labelled=n)[0] for bg, mine, n in parts]
        torch.cuda.synchronize()
        ms.append((time.perf_counter() - t0) * 1e3)
        losses.append(round(float(sum(s.item() for s in sums)) / max(1, sum(n for _, _, n in parts)), 5))
    best = min(ms[1:])
    print(json.dumps({"metric": "residual_training_epoch", "value": round(best, 3), "unit": "ms", "higher_is_better": False, "steps": len(parts),
                      "ms_per_step": round(best / len(parts), 4), "loss": losses, "dtype": args.dtype, "state_bits": args.bits,
                      "peak_gb": round(torch.cuda.max_memory_allocated() / 2 ** 30, 2),
                      "config": {"graph": cfg.name if hasattr(cfg, "name") else args.config, "nodes": g.n, "layers": L, "width": f, "norm": args.norm,
                                 "gate": not args.no_gate}}))


if __name__ == "__main__":
    main()
