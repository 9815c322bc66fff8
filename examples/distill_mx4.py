"""Fits a 4-bit output layer to a teacher's top logits, then serves single tokens from it.

The layer's master weight is an MC value of binary16 components.  Each step quantises it to
MXFP4, runs the layer on a batch of hidden states, takes the distillation loss and its gradient,
and adds the weight's gradient to the master (Grow-ExpN).  The upstream gradient of the loss
carries the step size, so the layer's backward pass returns the update itself.  With one
component an update below half a unit in the last place of a weight is lost; with two it is
kept.  At the end single rows go through the same 4-bit weight, as a decoding server would send
them.

    python examples/distill_mx4.py [--steps 300] [--master 2] [--nc 1]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2207_08867_amd as mcf


def split(x, nc):
    """nc binary16 components by successive rounding."""
    parts = []
    for _ in range(nc):
        parts.append(x.half())
        x = x - parts[-1].float()
    return torch.stack(parts)


def run(steps=300, master=2, nc=1, rows=512, hidden=256, vocab=2000, k=32, temperature=2.0, lr=4.0, seed=0):
    """Returns (the mean loss before every step, the share of tokens whose best logit is the teacher's)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    teacher = normal(vocab, hidden) / hidden ** 0.5 * 2.0
    x = normal(rows, hidden).half()
    t, ids = torch.topk(x.float() @ teacher.t(), k, dim=-1)
    t, ids = t.half(), ids.to(torch.int32)
    weight = split(teacher + normal(vocab, hidden) / hidden ** 0.5, master)
    g = torch.full((rows,), -lr / rows, device="cuda")
    losses = torch.empty(steps, device="cuda")
    for i in range(steps):
        w4 = mcf.mc_mx4_quantize(weight, nc=nc, x_mc=True)
        z = mcf.mc_mx4_linear_fwd(x, w4)
        loss, dz = mcf.mc_distill_fwd_bwd(z, ids, t, g, temperature=temperature)
        _, update, _ = mcf.mc_mx4_linear_bwd(x, w4, dz, dx=False, db=False)
        mcf.mc_add(weight, update, nc=master, y_mc=False, out=weight)
        losses[i] = loss.mean()
    w4 = mcf.mc_mx4_quantize(weight, nc=nc, x_mc=True)
    best = torch.stack([mcf.mc_mx4_linear_fwd(x[i:i + 1], w4)[0].argmax() for i in range(rows)])
    return losses.tolist(), (best == ids[:, 0]).float().mean().item()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--master", type=int, default=2, help="binary16 components of the master weight")
    ap.add_argument("--nc", type=int, default=1, help="MXFP4 components of the layer's weight")
    args = ap.parse_args()
    losses, agree = run(steps=args.steps, master=args.master, nc=args.nc)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {args.steps} steps; "
          f"{100 * agree:.1f}% of single tokens choose the teacher's best entry")


if __name__ == "__main__":
    main()
