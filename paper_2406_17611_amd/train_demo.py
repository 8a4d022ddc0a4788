"""Accuracy against communicated bytes on a labelled synthetic graph, for the settings Section V compares:
full communication, no communication, a fixed compression ratio and the variable schedule (Algorithm 1).

    python -m paper_2406_17611_amd.train_demo [--steps 150] [--blocks 8] [--block-size 2000] [--parts 8] [--max-norm N]

The graph is a stochastic block model whose blocks are the classes, dealt to random equal partitions (so most
neighbours of a node are remote); features carry a weak class signal under unit noise, so that aggregating over
neighbours, i.e. communicating, matters. Prints one JSON line per setting: held-out accuracy and the bytes
handed off between partitions (forward + backward) along the run; with --max-norm, gradients limited to that norm, the norm
of the last step's as well. All arithmetic runs in libvarco's kernels.
"""
from __future__ import annotations

import argparse
import json
import sys

import torch

from . import binding as vb
from . import synth
from .runner import PartitionedNetwork


def run(task, name, ratio_of_step, steps, lr, every, max_norm=None):
    host = vb.partition_build(task.graph.n, task.graph.rowptr, task.graph.colidx, task.graph.vals, task.part, task.n_parts)
    net = PartitionedNetwork(host, task.widths, task.conv, synth.MASK_KEY)
    L = net.L
    net.set_inputs(task.features)
    net.set_labels(task.labels, task.train)
    net.set_weights([synth.glorot(task.widths[l], task.widths[l + 1], synth.SEED_WEIGHT, 2 * l) for l in range(L)],
                    [synth.glorot(task.widths[l], task.widths[l + 1], synth.SEED_WEIGHT, 2 * l + 1) for l in range(L)])
    def traffic():
        st = net.ctx.stats()
        return (sum(st["fwd_elems"]) + sum(st["bwd_elems"])) * st["bytes_per_elem"]

    curve, sent = [], 0
    for step in range(steps):
        ratio = ratio_of_step(step)
        before = traffic()
        totals = net.train_step(step, ratio, lr, max_norm=max_norm)
        sent += traffic() - before               # training traffic only; the evaluation passes below are not counted
        if (step + 1) % every == 0 or step == steps - 1:
            torch.cuda.synchronize()
            risk = float(totals.cpu()[0])
            net.forward(10**6 + step, ratio)     # held-out nodes, same exchange setting, a step index of its own
            t = net.loss(train=False, with_gradient=False)
            torch.cuda.synchronize()
            curve.append({"step": step + 1, "train_risk": round(risk, 4),
                          "test_accuracy": round(float(t.cpu()[1]) / net.n_test, 4), "bytes_sent": int(sent),
                          **({} if max_norm is None else {"gradient_norm": round(float(net.gradient_norm.cpu()[0]), 5)})})
    return {"setting": name, "final_test_accuracy": curve[-1]["test_accuracy"], "bytes_sent": curve[-1]["bytes_sent"],
            "curve": curve}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--blocks", type=int, default=8)
    ap.add_argument("--block-size", type=int, default=2000)
    ap.add_argument("--parts", type=int, default=8)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--c-max", type=int, default=32)
    ap.add_argument("--max-norm", type=float, default=None)
    args = ap.parse_args()
    assert torch.cuda.is_available(), "train_demo needs a GPU"
    task = synth.labelled_sbm(n_blocks=args.blocks, block_size=args.block_size, p_in=8.0 / args.block_size,
                              p_out=1.0 / args.block_size, width=32, hidden=64, signal=0.3, n_parts=args.parts, conv="sage")
    every = max(1, args.steps // 10)
    K = args.steps
    settings = [
        ("full communication", lambda s: (1, 1)),
        ("no communication", lambda s: (1, 0)),
        ("fixed ratio 4", lambda s: (4, 1)),
        (f"variable: linear, c_max {args.c_max}, c_min 1, slope 2",
         lambda s: vb.schedule_ratio(vb.SCHED_LINEAR, s, K, args.c_max, 1, 2)),
        (f"variable: exponential base 2, c_max {args.c_max}", lambda s: vb.schedule_ratio(vb.SCHED_EXPONENTIAL, s, K, args.c_max, 1, 2)),
    ]
    for name, sched in settings:
        print(json.dumps(run(task, name, sched, args.steps, args.lr, every, args.max_norm)), flush=True)


if __name__ == "__main__":
    sys.exit(main())
