"""Quantise a gated feed-forward block, train it on, and serve it in 8 bits.

The gate and up projections are quantised at three bits as a controller would have it done.  The fake-quantised weights then are
the start of a short training run that follows the block as it was: windq_gated_forward keeps both products,
windq_gated_backward gives the weights' gradients, and windq_adamw_step steps 32-bit parameters with 16-bit copies that the next
pass reads.  Last, the trained block and its down projection are quantised row by row and serve a batch of single tokens:
windq_quantize_rows, windq_gated_int8_forward, windq_quantize_rows, windq_int8_forward.

    python examples/feed_forward.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_26660_b200 as wq   # noqa: E402
import windq_synth as ws             # noqa: E402

C, F, G, TOKENS, STEPS = 512, 1408, 128, 384, 40


def quantised(ctx, W, s):
    """The fake-quantised weight of a plan with three bits for every unit."""
    grid = torch.from_numpy(ws.clip_grid(20)).cuda()
    fit = wq.windq_fit_eval(ctx, W, G, s, grid)
    actions = torch.full((C // G,), 3, dtype=torch.uint8, device="cuda")
    bits = wq.windq_effective_bits(ctx, actions, W.shape[0], G)
    codes = torch.empty(int(bits["code_offsets"][-1]), dtype=torch.uint8, device="cuda")
    return wq.windq_apply_plan(ctx, W, G, s, grid, actions, bits["code_offsets"], codes, fit["clip_idx"])["wq"]


def main(verbose=True):
    torch.manual_seed(0)
    ctx = wq.windq_create()
    teacher = [(2.0 * ws.weights(F, C, k, "student_t", device="cuda").float()).half() for k in (1, 2)]
    down = ws.weights(C, F, 3, "student_t", device="cuda")
    s = wq.windq_act_stats(ctx, torch.randn(512, C, device="cuda").half())
    copies = [quantised(ctx, W, s) for W in teacher]              # what the passes read
    master = [W.float() for W in copies]                          # what the optimiser steps
    grads = [torch.zeros_like(W) for W in copies]
    zeros = lambda: [torch.zeros_like(W) for W in master]         # noqa: E731
    tensors = wq.AdamwTensors(master, grads, zeros(), zeros(), copies=copies)

    first, losses = None, []
    for step in range(1, STEPS + 1):
        X = torch.randn(TOKENS, C, device="cuda").half()
        want = wq.windq_gated_forward(ctx, X, *teacher)["h"].float()
        now = wq.windq_gated_forward(ctx, X, *copies, want_saved=True)
        miss = now["h"].float() - want
        losses.append(float(miss.square().mean()))
        dH = (miss * (2.0 / TOKENS)).half()
        if first is None:
            first = dict(X=X, Wg=copies[0].clone(), Wu=copies[1].clone(), dH=dH)
        wq.windq_gated_backward(ctx, X, *copies, dH, gate=now["gate"], up=now["up"], want_dx=False, out=dict(dWg=grads[0], dWu=grads[1]))
        if step == 1:
            first |= dict(dWg=grads[0].clone(), dWu=grads[1].clone())
        wq.windq_adamw_step(ctx, tensors, step=step, lr=2e-3)

    # serving: codes of the trained weights, made once, and of every batch of tokens.  They are a second rounding, with one scale a row:
    # a plan's own codes have a zero point and a scale for each group, which no integer product reads.
    coded = [wq.windq_quantize_rows(ctx, W) for W in (*copies, down)]
    X = torch.randn(6, C, device="cuda").half()
    x = wq.windq_quantize_rows(ctx, X)
    h = wq.windq_gated_int8_forward(ctx, x["codes"], x["scale"], *(t for w in coded[:2] for t in (w["codes"], w["scale"])))
    q = wq.windq_quantize_rows(ctx, h)
    Y = wq.windq_int8_forward(ctx, q["codes"], q["scale"], coded[2]["codes"], coded[2]["scale"])
    if verbose:
        print("loss %.5f -> %.5f in %d steps" % (losses[0], losses[-1], STEPS))
        full = wq.windq_gated_forward(ctx, X, *copies)["h"].float() @ down.float().T
        print("served in 8 bits: %.4f off the 16-bit block, relative" % float((Y.float() - full).norm() / full.norm()))
    served = dict(X=X, weights=(*copies, down), H=h, Y=Y)
    wq.windq_destroy(ctx)
    return losses, first, served


if __name__ == "__main__":
    main()
