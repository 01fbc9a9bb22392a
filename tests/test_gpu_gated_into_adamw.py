"""Gradients that windq_gated_backward allocates itself go into the optimiser as they are."""
import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,F,C,dtype", [(30, 96, 1000, HALF), (200, 520, 1000, BF), (300, 1, 72, HALF), (65, 100, 8, BF), (700, 1304, 1304, HALF),
                                         (0, 40, 24, HALF), (50, 64, 512, BF)])
def test_new_gradients_step_the_weights(wq, ctx, T, F, C, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(C)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X, Wg, Wu, dH = r(T, C).to(dtype), (0.1 * r(F, C)).to(dtype), (0.1 * r(F, C)).to(dtype), r(T, 8 * (-(-F // 8))).to(dtype)[:, :F]

    def stepped(**out):
        d = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, **out)
        grads = [d["dWg"], d["dWu"]]
        assert all(t.is_contiguous() and t.view(-1).shape == (F * C,) for t in grads)
        master = [Wg.float(), Wu.float()]
        tensors = wq.AdamwTensors(master, grads, [torch.zeros_like(w) for w in master], [torch.zeros_like(w) for w in master])
        wq.windq_adamw_step(ctx, tensors, step=1, lr=1e-2)
        return grads + master

    a = stepped()
    b = stepped(out=dict(dWg=torch.empty((F, C), dtype=dtype, device="cuda"), dWu=torch.empty((F, C), dtype=dtype, device="cuda")))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert T == 0 or bool((a[2] != Wg.float()).any())


def test_strides_of_new_outputs(wq, ctx):  # noqa: F811
    """As the docstrings have them: rows that are no multiple of 32 bytes, the next multiple of 128 bytes apart."""
    X, W = torch.randn((40, 1000), device="cuda").half(), torch.randn((1000, 1000), device="cuda").half()
    f = wq.windq_gated_forward(ctx, X, W, W, want_saved=True)
    d = wq.windq_gated_backward(ctx, X, W, W, f["h"], gate=f["gate"], up=f["up"])
    q = wq.windq_quantize_rows(ctx, X, want_values=True)
    w = wq.windq_quantize_rows(ctx, W)
    y = wq.windq_int8_forward(ctx, q["codes"], q["scale"], w["codes"], w["scale"])
    h = wq.windq_gated_int8_forward(ctx, q["codes"], q["scale"], w["codes"], w["scale"], w["codes"], w["scale"])
    assert [t.stride() for t in (f["h"], f["gate"], f["up"], d["dx"], q["values"], q["codes"], y, h)] == [(1024, 1)] * 8
    assert d["dWg"].stride() == d["dWu"].stride() == (1000, 1)
    odd = wq.windq_gated_backward(ctx, W[:, :999], W[:, :999], W[:, :999], W[:, :1000])
    assert odd["dWg"].stride() == odd["dWu"].stride() == (1024, 1)
