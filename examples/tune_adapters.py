"""Quantise a layer, tune two low-rank adapters beside it, and serve both in one batch.

The layer's weight is scored and quantised at two bits as a controller would have it done; two adapters then learn what
quantisation lost -- one for the layer as it was, one for the layer after a small change, as fine-tuning would make it --
from batches in which the two tasks' sequences follow one another.  Their gradients come from windq_lora_backward, the
step is windq_adamw_step with 8-bit states, which also writes the 16-bit copies the next forward pass reads.  Last, single
tokens of both tasks are served together, with one that has no adapter.

    python examples/tune_adapters.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_26660_b200 as wq   # noqa: E402
import windq_synth as ws             # noqa: E402

R, C, G, RANK, TOKENS, STEPS = 512, 1024, 128, 16, 640, 60


def quantised(ctx, W, X):
    """The fake-quantised weight of a plan with two bits for every unit."""
    s = wq.windq_act_stats(ctx, X)
    grid = torch.from_numpy(ws.clip_grid(20)).cuda()
    fit = wq.windq_fit_eval(ctx, W, G, s, grid)
    actions = torch.full((C // G,), 4, dtype=torch.uint8, device="cuda")
    bits = wq.windq_effective_bits(ctx, actions, R, G)
    codes = torch.empty(int(bits["code_offsets"][-1]), dtype=torch.uint8, device="cuda")
    return wq.windq_apply_plan(ctx, W, G, s, grid, actions, bits["code_offsets"], codes, fit["clip_idx"])["wq"]


def zeros_like_states(params):
    """Empty 8-bit states of some parameters: codes and scales, all zero."""
    blocks = lambda p: torch.zeros(-(-p.numel() // wq.ADAMW_BLOCK), device="cuda")  # noqa: E731
    return dict(m=[torch.zeros(p.shape, dtype=torch.int8, device="cuda") for p in params],
                v=[torch.zeros(p.shape, dtype=torch.uint8, device="cuda") for p in params],
                m_scale=[blocks(p) for p in params], r_scale=[blocks(p) for p in params])


def main(verbose=True):
    torch.manual_seed(0)
    ctx = wq.windq_create()
    W = ws.weights(R, C, 1, "student_t", device="cuda")
    calibration = torch.randn(512, C, device="cuda").half()
    Wq = quantised(ctx, W, calibration)
    changed = (W.float() + 0.01 * torch.randn(R, 4, device="cuda") @ torch.randn(4, C, device="cuda")).half()
    teachers = (W.float(), changed.float())

    # fp32 master adapters and the 16-bit ones the layer computes with; B starts at zero, so the adapters start as nothing
    A = torch.randn(2, RANK, C, device="cuda") / C ** 0.5
    B = torch.zeros(2, R, RANK, device="cuda")
    A16, B16 = A.half(), B.half()
    scaling = torch.full((2,), 2.0, device="cuda")
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    adapters = wq.AdamwTensors([A, B], [dA, dB], copies=[A16, B16], **zeros_like_states([A, B]))

    half = TOKENS * 2 // 3   # the two tasks' sequences are of unequal length
    ids = torch.tensor([0] * half + [1] * (TOKENS - half), dtype=torch.int32, device="cuda")
    losses = []
    for step in range(1, STEPS + 1):
        X = torch.randn(TOKENS, C, device="cuda").half()
        want = torch.cat([X[:half].float() @ teachers[0].T, X[half:].float() @ teachers[1].T])
        Y = wq.windq_lora_forward(ctx, X, Wq, A16, B16, scaling, ids)
        miss = Y.float() - want
        losses.append(float(miss.square().mean()))
        wq.windq_lora_backward(ctx, X, Wq, A16, B16, scaling, ids, (miss * (2.0 / TOKENS)).half(), want_dx=False,
                               out=dict(dA=dA, dB=dB))
        wq.windq_adamw_step(ctx, adapters, step=step, lr=5e-3, weight_decay=0.0)

    # serving: single tokens, each with its request's adapter (-1: the shared layer alone)
    X = torch.randn(6, C, device="cuda").half()
    ids = torch.tensor([0, 1, -1, 1, 0, -1], dtype=torch.int32, device="cuda")
    Y = wq.windq_lora_forward(ctx, X, Wq, A16, B16, scaling, ids).float()
    served = []
    for t, a in enumerate(ids.tolist()):
        want = X[t].float() @ teachers[max(a, 0)].T
        served.append(float((Y[t] - want).square().mean() / want.square().mean()))
    if verbose:
        print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], STEPS))
        for a, e in zip(ids.tolist(), served):
            print("  served with %s: relative squared error %.4f" % ("adapter %d" % a if a >= 0 else "no adapter", e))
    wq.windq_destroy(ctx)
    return losses, ids.tolist(), served


if __name__ == "__main__":
    main()
