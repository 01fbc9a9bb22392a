"""A decode loop without a wait: every round quantises other tokens into the same codes and scales, and a product reads them right
behind.  The kernels overlap, so a product may be on an SM while its tokens' scales are still those of the round before."""
import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,R,C,dtype", [(1, 2048, 2048, HALF), (3, 300, 520, BF), (40, 4096, 1024, BF), (64, 128, 8192, HALF), (65, 1000, 1000, HALF),
                                         (128, 2048, 512, BF), (300, 2048, 2048, HALF), (1000, 1024, 256, BF)])
def test_tokens_change_in_place(wq, ctx, T, R, C, dtype, gated):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w, v = (wq.windq_quantize_rows(ctx, 0.1 * r(R, C).to(dtype)) for _ in range(2))
    tokens = [(size * r(T, C)).to(dtype) for size in (1.0, 16.0, 1 / 16)]      # a scale of another round is far off

    def product(x):
        if gated:
            return wq.windq_gated_int8_forward(ctx, x["codes"], x["scale"], w["codes"], w["scale"], v["codes"], v["scale"], dtype=dtype)
        return wq.windq_int8_forward(ctx, x["codes"], x["scale"], w["codes"], w["scale"], dtype=dtype)

    want = []
    for X in tokens:
        x = wq.windq_quantize_rows(ctx, X)
        torch.cuda.synchronize()
        want.append(product(x))
        torch.cuda.synchronize()
    x = wq.windq_quantize_rows(ctx, tokens[0])
    got = []
    for k in range(200):
        wq.windq_quantize_rows(ctx, tokens[k % 3], out=x)
        got.append(product(x))
    for k, y in enumerate(got):
        assert torch.equal(y, want[k % 3]), k


def test_weights_and_their_scales_change_in_place(wq, ctx):  # noqa: F811
    """The scales of the outputs, too, are those that the kernel before leaves."""
    g = torch.Generator(device="cuda").manual_seed(5)
    T, R, C = 20, 2048, 1024
    x = wq.windq_quantize_rows(ctx, torch.randn((T, C), generator=g, device="cuda").half())
    weights = [size * torch.randn((R, C), generator=g, device="cuda").half() for size in (0.1, 1.0, 8.0)]
    want = []
    for W in weights:
        w = wq.windq_quantize_rows(ctx, W)
        torch.cuda.synchronize()
        want.append(wq.windq_int8_forward(ctx, x["codes"], x["scale"], w["codes"], w["scale"]))
        torch.cuda.synchronize()
    w = wq.windq_quantize_rows(ctx, weights[0])
    got = []
    for k in range(90):
        wq.windq_quantize_rows(ctx, weights[k % 3], out=w)
        got.append(wq.windq_int8_forward(ctx, x["codes"], x["scale"], w["codes"], w["scale"]))
    for k, y in enumerate(got):
        assert torch.equal(y, want[k % 3]), k
