"""Gradients of the gated block in fp16 where a value is not finite: it spoils its own token and output, and nothing else."""
import pytest
import torch

from test_gpu_gated import exact_gradients
from test_gpu_quantize_rows import HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu

# few tokens, two terms on pairs of thread blocks, one term
SIZES = [(40, 256, 128), (500, 256, 128), (700, 1304, 1304)]


@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("small", [True, False])
@pytest.mark.parametrize("T,F,C", SIZES)
def test_the_range_of_the_others(wq, ctx, T, F, C, small, bad):  # noqa: F811
    """dG and dU of the other tokens are below fp16's numbers, or beyond them, as they would be stored without a power of two."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    g, u = r(T, F).half(), (r(T, F) * (0.001 if small else 2000)).half()
    dH = (r(T, F) * (1e-5 if small else 300)).half()
    X = (r(T, C) * (10000 if small else 1e-3)).half()
    Wg, Wu = ((r(F, C) * (10000 if small else 1e-4)).half() for _ in range(2))
    t, f = T - 3, 50
    dH[t, f] = 0
    want, _, _ = exact_gradients(X, Wg, Wu, dH, g, u, "silu")
    dH[t, f] = float(bad)
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=g, up=u)
    for k, row in (("dx", t), ("dWg", f), ("dWu", f)):
        assert not bool(got[k][row].isfinite().any()), k
        others = torch.arange(want[k].shape[0], device="cuda") != row
        a, b = got[k][others].double(), want[k][others]
        fits = b.abs() < 60000
        assert float(b.abs().max()) > 1e-3 and bool(a[fits].isfinite().all()), k
        # a rounding of each term and one of the result, independent of one another: below twice a rounding in the mean
        off = (a - b)[fits].norm() / b[fits].norm()
        assert float(off) < 2 * 2.0 ** -11, (k, float(off))


def test_no_finite_value_at_all(wq, ctx):  # noqa: F811
    X, W = torch.ones((70, 64), dtype=HALF, device="cuda"), torch.ones((72, 64), dtype=HALF, device="cuda")
    g = torch.ones((70, 72), dtype=HALF, device="cuda")
    got = wq.windq_gated_backward(ctx, X, W, W, torch.full_like(g, float("nan")), gate=g, up=g)
    assert all(bool(got[k].isnan().all()) for k in got)
