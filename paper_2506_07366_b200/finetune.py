"""Example: fine-tuning one MoE layer with MoeTrainLayer.

    python -m paper_2506_07366_b200.finetune [--steps N] [--lr X]

A layer of the "tiny" workload's shape learns to reproduce another one of the same shape (other experts, same router at the
start) on two batches of seeded synthetic tokens: mean squared error, fp32 master copies of the weights, and steps that move
each of them by lr times its root mean square along its gradient.  Every batch is planned from the histogram of the batch
before it, as in inference.  Prints the loss of every step's batch, relative to the mean square of what it should be.
"""
from __future__ import annotations

import argparse
import dataclasses

import torch

from . import workloads as wl
from .binding import Shape
from .layer import ROW_ALIGN, MoeLayer, MoeTrainLayer


def finetune(steps: int = 30, lr: float = 0.02, device: str = "cuda", log=print) -> list[float]:
    w = dataclasses.replace(wl.WORKLOADS["tiny"], sigma_x=1.0, S=10)
    shape = Shape(w.T, w.D, w.F, w.E, w.K, w.S, w.gate_mode, ROW_ALIGN)
    wr, bias = wl.router(w, device)
    teacher = MoeLayer(shape, wr, bias, *wl.expert_weights(w, device))
    student_w = dataclasses.replace(w, number=w.number + 50)
    names = ("w_gate", "w_up", "w_down", "w_router", "bias")
    start = (*wl.expert_weights(student_w, device), wr.clone(), bias.clone())
    master = {n: v.float() for n, v in zip(names, start)}
    student = MoeTrainLayer(shape, start[3], start[4], *start[:3])
    pred = torch.full((w.E,), w.R // w.E, dtype=torch.int32, device=device)
    batches = [wl.redraw_rows(w, w.T, i, device) for i in range(2)]
    losses = []
    for step in range(steps):
        x = batches[step % len(batches)]
        teacher.plan(pred)
        student.plan(pred)
        want = teacher.forward(x).float()
        off, square = student.forward_train(x).float() - want, want.square().sum()
        losses.append(float(off.square().sum() / square))
        grads = student.backward((off * (2 / square)).to(torch.bfloat16))
        for n, m in master.items():
            g = grads[n].float()
            m -= g * (lr * m.square().mean().sqrt() / g.square().mean().sqrt().clamp_min(1e-30))
            getattr(student, n).copy_(m)
        pred = student.hist.clone()
        student.ctx.check_status()
        log(f"step {step:3d}  loss {losses[-1]:.4f}")
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=0.02)
    a = ap.parse_args()
    finetune(a.steps, a.lr)


if __name__ == "__main__":
    main()
