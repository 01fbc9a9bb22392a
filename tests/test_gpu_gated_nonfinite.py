"""Gradients of the gated block where a value is not finite: it spoils its own token and output, and nothing else; and gates so far out
that the forward pass leaves infinities of them, which are shut all the same."""
import pytest
import torch

from test_gpu_gated import exact_gradients
from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

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


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [20, 300])
def test_shut_gates_beyond_fp16(wq, ctx, T, act):  # noqa: F811
    """g = -120000 in every second output, u = +-120000 in every third: kept as infinities, while H is 0 and so are dG and dU."""
    F, C = 96, 64
    X = torch.zeros((T, C), dtype=HALF, device="cuda")
    X[:, 0] = 2
    Wg, Wu = torch.full((F, C), 0.5, dtype=HALF, device="cuda"), torch.full((F, C), 0.25, dtype=HALF, device="cuda")
    Wg[:, 0], Wu[:, 0] = 20, 1                            # open gates, g = 40
    Wg[::2, 0] = -60000
    Wu[::6, 0], Wu[2::6, 0] = 60000, -60000               # of shut gates alone
    f = wq.windq_gated_forward(ctx, X, Wg, Wu, activation=act, want_saved=True)
    assert bool((f["gate"][:, ::2] == float("-inf")).all()) and bool((f["up"][:, ::6] == float("inf")).all())
    assert bool((f["h"][:, ::2] == 0).all()) and bool((f["h"][:, 1::2] == 80).all())
    dH = torch.ones((T, F), dtype=HALF, device="cuda")
    for saved in (dict(gate=f["gate"], up=f["up"]), {}):
        got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, activation=act, **saved)
        # open gates: dG = u = 2, dU = g = 40 (exp(-40) is below a rounding), sums of integers
        assert bool((got["dWg"][::2] == 0).all()) and bool((got["dWu"][::2] == 0).all())
        assert bool((got["dWg"][1::2, 0] == 4 * T).all())
        assert torch.equal(got["dWu"][1::2, 0], torch.full((F // 2,), 80.0 * T, device="cuda").half())
        assert bool((got["dx"][:, 1:] == 48 * (2 * 0.5 + 40 * 0.25)).all()) and bool((got["dx"][:, 0] == 48 * (2 * 20 + 40)).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_what_a_shut_gate_does_not_hide(wq, ctx, dtype, act):  # noqa: F811
    """A NaN in the gate, in up or in the gradient of H is a mistake of the caller's and stays visible."""
    T, F, C = 7, 64, 64
    X, W = torch.ones((T, C), dtype=dtype, device="cuda"), torch.ones((F, C), dtype=dtype, device="cuda")
    for name in ("gate", "up", "dH"):
        a = dict(gate=torch.full((T, F), float("-inf"), dtype=dtype, device="cuda"), up=torch.full((T, F), float("inf"), dtype=dtype, device="cuda"),
                 dH=torch.ones((T, F), dtype=dtype, device="cuda"))
        a[name][2, 5] = float("nan")
        got = wq.windq_gated_backward(ctx, X, W, W, a.pop("dH"), activation=act, **a)
        rows = torch.arange(T, device="cuda") != 2
        assert bool(got["dx"][2].isnan().all()) and bool((got["dx"][rows] == 0).all())
        outputs = torch.arange(F, device="cuda") != 5
        assert bool((got["dWg"][outputs] == 0).all()) and bool((got["dWu"][outputs] == 0).all())
        assert bool(got["dWg"][5].isnan().all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [20, 300])
def test_tokens_without_a_gradient(wq, ctx, T, act):  # noqa: F811
    """Padding, and tokens outside the loss: their gates and ups may be beyond fp16, their dH is 0, and so is what they add."""
    F, C = 96, 64
    gen = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    X, Wg, Wu = r(T, C).half(), (0.1 * r(F, C)).half(), (0.1 * r(F, C)).half()
    Wg[:, 0], Wu[:, 0] = 30, -30
    X[:, 0] = 0
    masked = torch.arange(T, device="cuda") % 3 == 1
    X[masked, 0] = 30000                                  # g = 900000, u = -900000
    dH = r(T, F).half()
    dH[masked] = 0
    f = wq.windq_gated_forward(ctx, X, Wg, Wu, activation=act, want_saved=True)
    assert bool(f["gate"][masked].isinf().all()) and bool(f["up"][masked].isinf().all()) and bool(f["h"][~masked].isfinite().all())
    kept = wq.windq_gated_backward(ctx, X[~masked].contiguous(), Wg, Wu, dH[~masked].contiguous(), activation=act)
    for saved in (dict(gate=f["gate"], up=f["up"]), {}):
        got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, activation=act, **saved)
        assert bool((got["dx"][masked] == 0).all())
        # the same sums beside zeros: what differs is where the tensor cores cut them off, below a rounding of the result
        for a, b in ((got["dx"][~masked], kept["dx"]), (got["dWg"], kept["dWg"]), (got["dWu"], kept["dWu"])):
            assert bool(a.isfinite().all()) and float((a.double() - b.double()).norm() / b.double().norm()) < 2.0 ** -11
