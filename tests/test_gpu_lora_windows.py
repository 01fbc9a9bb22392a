"""Gradients over more tokens than one look-up takes (4096), with the largest low-rank values late, early or in the middle:
the fp16 terms of S are scaled by the largest so far, and the sums are rescaled where a later window has a larger one."""
import pytest
import torch

from test_gpu_lora import BF, HALF, backward, ctx, exact, gen, inputs, padded, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [HALF, BF])
@pytest.mark.parametrize("order", ["rising", "falling", "peak"])
@pytest.mark.parametrize("T,R,C,r,n,kind", [(9000, 264, 136, 16, 2, "mixed"), (13000, 40, 264, 40, 3, "segments"), (8200, 72, 72, 8, 1, "one")])
def test_windows_of_unequal_size(wq, ctx, T, R, C, r, n, kind, order, dt):  # noqa: F811
    # integers times a power of two that changes with the window; sums of all sizes are exact in binary32 over four steps
    q, dY = inputs(T, R, C, r, n, dt, kind, seed=80)
    window = torch.arange(T, device="cuda") // 4096
    last = int(window[-1])
    step = {"rising": window, "falling": last - window, "peak": 2 - 2 * (window - 1).abs()}[order]
    size = torch.exp2(-3.0 + step.float())[:, None]
    q["X"] = (q["X"].float() * (torch.rand((T, 1), generator=gen(T), device="cuda") < 0.02)).to(dt)     # few tokens, or the sums outgrow 24 bits
    dY = padded((dY.float() * size).to(dt))
    want, back = exact(q, dY), backward(wq, ctx, q, dY)
    assert torch.equal(back["dx"], want["dx"].to(dt))
    assert torch.equal(back["dA"], want["dA"].float()) and torch.equal(back["dB"], want["dB"].float())
    # and real values, relative to the whole: far apart between windows
    q, dY = inputs(T, R, C, r, n, dt, kind, seed=81, integers=False)
    dY = padded((dY.float() * torch.exp2(3.0 * step.float() - 12)[:, None]).to(dt))
    q["X"] = (q["X"].float() * torch.exp2(-2.0 * step.float())[:, None]).to(dt)
    want, back = exact(q, dY), backward(wq, ctx, q, dY, want_dx=False)
    for k in ("dA", "dB"):
        for a in range(n):
            assert float((back[k][a].double() - want[k][a]).norm()) <= 1e-5 * float(want[k][a].norm()), (k, a)
