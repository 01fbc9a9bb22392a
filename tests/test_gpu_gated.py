"""The gated feed-forward block, its gradients, and its 8-bit form.

Most cases are small integers: the products then are exact in binary32, so g and u are, and H can be told to a rounding.  With
a gate of 32 or more the logistic function is one in binary32 (exp(-32) is below 2^-46) and its slope zero, so dG = dH u and
dU = dH g are integers of a few bits, every sum is exact and the gradients must be the 64-bit ones rounded once."""
import math

import pytest
import torch

from test_gpu_int8_forward import codes, product, scales
from test_gpu_quantize_rows import BF, HALF, ctx, padded, wq  # noqa: F401

pytestmark = pytest.mark.gpu

NAN = float("nan")
# Beside the last rounding H carries: exp's argument rounded a few times (|y| 2^-24 each, and what exp leaves of binary32 has
# |y| < 90) and the function's own few ulp, below 2^-17 together, then the quotient and three products (2^-21)
FAST = 2.0 ** -16


def integers(shape, seed, dtype, low=-3, high=4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(low, high, shape, generator=g, device="cuda").to(dtype)


def activation(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))   # (1 + tanh would cancel)


def slope(g, act):
    with torch.enable_grad():
        x = g.detach().clone().requires_grad_(True)
        return torch.autograd.grad(activation(x, act).sum(), x)[0]


def near(got, want, dtype):
    """got is want (64 bits), off by at most FAST and a rounding to dtype."""
    u = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).tiny * u                     # half a step of the subnormal numbers
    off = (got.double() - want).abs()
    assert bool((off <= (u * (1 + FAST) + FAST) * want.abs() + tiny).all()), float((off / want.abs().clamp(min=1e-9)).max())


def block(T, F, C, dtype, seed):
    """Tokens and weights whose products are integers, divided down to where the gate is neither open nor shut."""
    return integers((T, C), seed, dtype), integers((F, C), seed + 1, dtype) / 16, integers((F, C), seed + 2, dtype) / 16


SIZES = [(1, 64, 64), (1, 1, 1), (2, 65, 72), (16, 128, 1000), (17, 333, 130), (64, 1000, 264), (100, 700, 515), (200, 129, 2048),
         (256, 512, 96), (257, 512, 96), (320, 320, 320), (321, 320, 320), (500, 1027, 200), (1025, 264, 1032), (2300, 2048, 64), (300, 96, 8192),
         (400, 70, 8192)]


@pytest.mark.parametrize("dtype,act", [(HALF, "silu"), (BF, "gelu")])
@pytest.mark.parametrize("T,F,C", SIZES)
def test_forward(wq, ctx, T, F, C, dtype, act):  # noqa: F811
    X, Wg, Wu = block(T, F, C, dtype, T + F)
    g, u = X.double() @ Wg.double().T, X.double() @ Wu.double().T
    outs = {k: padded(torch.zeros((T, F), dtype=dtype, device="cuda"), 8, 3.0) for k in ("h", "gate", "up")}
    got = wq.windq_gated_forward(ctx, padded(X, 8, NAN)[0], padded(Wg, 8, NAN)[0], padded(Wu, 8, NAN)[0], activation=act, want_saved=True,
                                 out={k: v[0] for k, v in outs.items()})
    assert torch.equal(got["gate"], g.to(dtype)) and torch.equal(got["up"], u.to(dtype))
    near(got["h"], activation(g, act) * u, dtype)
    assert all(bool((whole[:, F:] == 3).all()) for _, whole in outs.values())
    bare = wq.windq_gated_forward(ctx, padded(X, 8, NAN)[0], padded(Wg, 8, NAN)[0], padded(Wu, 8, NAN)[0], activation=act)
    assert torch.equal(bare["h"], got["h"]) and bare["gate"] is None and bare["up"] is None


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_gates_far_out(wq, ctx, dtype, act):  # noqa: F811
    """Gates from -1000 to 1000, where exponentials leave binary32: H is 0 or g u."""
    C, F = 64, 40
    X = torch.zeros((30, C), dtype=dtype, device="cuda")
    X[:, 0], X[:, 1] = 1, 1
    Wg, Wu = torch.zeros((F, C), dtype=dtype, device="cuda"), torch.zeros((F, C), dtype=dtype, device="cuda")
    Wg[:, 0], Wu[:, 1] = torch.linspace(-1000, 1000, F, device="cuda").to(dtype), 2
    for T in (30, 600):
        got = wq.windq_gated_forward(ctx, X[:1].expand(T, C).contiguous(), Wg, Wu, activation=act)["h"]
        g = Wg[:, 0].double()
        want = (activation(g, act) * 2).expand(T, F)
        off = (got.double() - want).abs()
        assert bool((off <= 2 * torch.finfo(dtype).eps * want.abs() + 1e-6).all())
        assert bool(got.isfinite().all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [3, 70])
def test_gates_of_any_size_in_bf16(wq, ctx, T, act):  # noqa: F811
    """Gates whose squares and cubes leave binary32: open ones pass u on, shut ones nothing, and so do their gradients."""
    C = F = 8
    X = torch.zeros((T, C), dtype=BF, device="cuda")
    X[:, 0], X[:, 1] = 1, 1
    Wg, Wu = torch.zeros((F, C), dtype=BF, device="cuda"), torch.zeros((F, C), dtype=BF, device="cuda")
    Wg[:, 0] = torch.tensor([1e10, -1e10, 1e20, -1e20, 1e36, -1e36, 200, -200], dtype=BF)
    Wu[:, 1] = 2
    f = wq.windq_gated_forward(ctx, X, Wg, Wu, activation=act, want_saved=True)
    opened = Wg[:, 0] > 0
    assert torch.equal(f["h"], torch.where(opened, 2 * Wg[:, 0], 0).expand(T, F))
    dH = torch.ones((T, F), dtype=BF, device="cuda")
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=f["gate"], up=f["up"], activation=act, want_dx=False)
    assert torch.equal(got["dWg"][:, 0], torch.where(opened, 2.0 * T, 0).to(BF))          # dG = dH u act'(g), act' one or zero
    assert torch.allclose(got["dWu"][:, 1].float(), torch.where(opened, T * Wg[:, 0].float(), 0), rtol=2.0 ** -7, atol=1e-30)


@pytest.mark.parametrize("T", [65, 96, 113, 128, 129])
def test_from_few_tokens_to_many(wq, ctx, T):  # noqa: F811
    X, Wg, Wu = block(T, 300, 1000, BF, T)
    g, u = X.double() @ Wg.double().T, X.double() @ Wu.double().T
    got = wq.windq_gated_forward(ctx, X, Wg, Wu, want_saved=True)
    assert torch.equal(got["gate"], g.to(BF)) and torch.equal(got["up"], u.to(BF))
    near(got["h"], activation(g, "silu") * u, BF)
    x, wg, wu, s = codes((T, 1008), 1), codes((300, 1008), 2), codes((300, 1008), 3), scales(300, 2) * 0.05
    h = wq.windq_gated_int8_forward(ctx, x, scales(T, 1), wg, s, wu, s)
    near(h, activation(product(x, wg, scales(T, 1), s).double(), "silu") * product(x, wu, scales(T, 1), s).double(), HALF)


def exact_gradients(X, Wg, Wu, dH, g, u, act):
    x, dh, g, u = X.double(), dH.double(), g.double(), u.double()
    du, dg = dh * activation(g, act), dh * u * slope(g, act)
    return dict(dx=dg @ Wg.double() + du @ Wu.double(), dWg=dg.T @ x, dWu=du.T @ x), dg, du


@pytest.mark.parametrize("dtype,act", [(HALF, "gelu"), (BF, "silu")])
@pytest.mark.parametrize("T,F,C", SIZES)
def test_gradients_of_open_gates(wq, ctx, T, F, C, dtype, act):  # noqa: F811
    X, Wg, Wu = integers((T, C), T, dtype), integers((F, C), F, dtype), integers((F, C), C, dtype)
    g, u = integers((T, F), 5, dtype, 32, 64), integers((T, F), 6, dtype, -40, 41)
    dH = integers((T, F), 7, dtype, -2, 3)
    dg, du, x = dH.double() * u.double(), dH.double() * g.double(), X.double()
    want = dict(dx=dg @ Wg.double() + du @ Wu.double(), dWg=dg.T @ x, dWu=du.T @ x)
    outs = {k: padded(torch.zeros(shape, dtype=dtype, device="cuda"), 8, 3.0) for k, shape in (("dx", (T, C)), ("dWg", (F, C)), ("dWu", (F, C)))}
    args = [padded(t, 8, NAN)[0] for t in (X, Wg, Wu, dH)]
    saved = dict(gate=padded(g, 8, NAN)[0], up=padded(u, 8, NAN)[0])
    got = wq.windq_gated_backward(ctx, *args, **saved, activation=act, out={k: v[0] for k, v in outs.items()})
    for k in ("dx", "dWg", "dWu"):
        assert torch.equal(got[k], want[k].to(dtype)), k
        assert bool((outs[k][1][:, C:] == 3).all())
    only = wq.windq_gated_backward(ctx, *args, **saved, activation=act, want_dw=False)
    assert torch.equal(only["dx"], got["dx"]) and only["dWg"] is None
    only = wq.windq_gated_backward(ctx, *args, **saved, activation=act, want_dx=False)
    assert torch.equal(only["dWg"], got["dWg"]) and torch.equal(only["dWu"], got["dWu"]) and only["dx"] is None


def bound(dtype, want, terms):
    """dG and dU rounded once (u each, and FAST), the sums of K such terms cut off in binary32 (2^-23 of all terms an addition
    of 16 or 32 of them, below 2^-12 for the sizes here), the result rounded."""
    u = torch.finfo(dtype).eps / 2
    return (u + FAST + 2.0 ** -12) * terms * (1 + u) + u * want.abs() + torch.finfo(dtype).tiny * u


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("T,F,C", [(1, 200, 300), (50, 333, 520), (64, 5000, 4000), (300, 1000, 264), (700, 520, 1000), (65, 6000, 3000),
                                   (400, 2100, 1400)])
def test_gradients_against_the_formula(wq, ctx, T, F, C, dtype, act):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    X, Wg, Wu, dH = (padded(t.to(dtype), 8, NAN)[0] for t in (r(T, C), 0.1 * r(F, C), 0.1 * r(F, C), 0.1 * r(T, F)))
    f = wq.windq_gated_forward(ctx, X, Wg, Wu, activation=act, want_saved=True)
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=f["gate"], up=f["up"], activation=act)
    want, dg, du = exact_gradients(X, Wg, Wu, dH, f["gate"], f["up"], act)
    # cancelling inside act'(g) leaves an error relative to its parts, |s| + |g s (1 - s) y'|, which are below 3
    u = torch.finfo(dtype).eps / 2
    part = (3 * FAST) * (dH.double() * f["up"].double()).abs()
    adg, adu = dg.abs() + part / (u + FAST), du.abs()
    terms = dict(dx=adg @ Wg.double().abs() + adu @ Wu.double().abs(), dWg=adg.T @ X.double().abs(), dWu=adu.T @ X.double().abs())
    for k in want:
        off = (got[k].double() - want[k]).abs()
        assert bool((off <= bound(dtype, want[k], terms[k])).all()), k
        # a rounding of each term and one of the result, independent of one another: well below twice a rounding in the mean
        assert float(off.norm() / want[k].norm()) < 2 * u, k
        if T <= 64 or T * F * C <= 1 << 30:
            # two terms: what is left beside the last rounding, FAST and what the tensor cores cut off (together below 2^-14.5 of the
            # norm, fp16's rounding above 2^-12.5 of it), adds in squares, below 4 %
            assert float(off.norm()) < 1.04 * float((want[k].to(dtype).double() - want[k]).norm()), k
    again = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, activation=act)     # computed again from X
    for k in want:
        assert torch.equal(again[k], got[k]), k


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(wq, ctx, act):  # noqa: F811
    """The change of <dH, H> along directions in X, Wg and Wu, from central differences of the block in 64 bits."""
    T, F, C = 40, 96, 64
    gen = torch.Generator(device="cuda").manual_seed(9)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    X, Wg, Wu, dH = (t.half() for t in (r(T, C), 0.2 * r(F, C), 0.2 * r(F, C), r(T, F)))
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, activation=act)
    value = lambda x, a, b: (dH.double() * activation(x @ a.T, act) * (x @ b.T)).sum()  # noqa: E731
    at, step = [t.double() for t in (X, Wg, Wu)], 1e-5
    for k, name in enumerate(("dx", "dWg", "dWu")):
        along = torch.randn(at[k].shape, generator=gen, device="cuda", dtype=torch.float64)
        moved = lambda s: value(*(t + s * step * along if i == k else t for i, t in enumerate(at)))  # noqa: E731, B023
        difference = (moved(1) - moved(-1)) / (2 * step)
        # every entry of the gradient is off by less than a few roundings of its rms: their sum over n random directions by sqrt(n) of that
        n, rms = along.numel(), float(got[name].double().square().mean().sqrt())
        assert abs(float((got[name].double() * along).sum() - difference)) < 8 * 2.0 ** -11 * rms * n ** 0.5 + 1e-6 * abs(float(difference))


@pytest.mark.parametrize("T", [40, 500])
@pytest.mark.parametrize("small", [True, False])
def test_small_and_large_gradients_in_fp16(wq, ctx, T, small):  # noqa: F811
    """dG and dU below fp16's normal numbers, or beyond its largest, with weights that bring the results back."""
    F, C = 256, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    g, u = r(T, F).half(), (r(T, F) * (0.01 if small else 2000)).half()
    dH = (r(T, F) * (1e-5 if small else 300)).half()
    X = (r(T, C) * (1000 if small else 1e-3)).half()
    Wg, Wu = ((r(F, C) * (1000 if small else 1e-4)).half() for _ in range(2))
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=g, up=u)
    want, _, _ = exact_gradients(X, Wg, Wu, dH, g, u, "silu")
    for k in want:
        fits = want[k].abs() < 60000
        assert float(want[k].abs().max()) > 1e-3
        off = (got[k].double() - want[k])[fits].norm() / want[k][fits].norm()
        assert float(off) < 2 * 2.0 ** -11, (k, float(off))


@pytest.mark.parametrize("T", [40, 500])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_zero_and_nonfinite_gradients(wq, ctx, T, dtype):  # noqa: F811
    X, Wg, Wu = block(T, 96, 64, dtype, 2)
    g, u = integers((T, 96), 5, dtype), integers((T, 96), 6, dtype)
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, torch.zeros_like(g), gate=g, up=u)
    assert all(bool((got[k] == 0).all()) for k in got)
    dH = integers((T, 96), 7, dtype)
    dH[3, 50] = NAN
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=g, up=u)
    assert bool(got["dx"][3].isnan().all()) and int(got["dx"].isnan().any(dim=1).sum()) == 1
    assert bool(got["dWg"][50].isnan().all()) and int(got["dWg"].isnan().any(dim=1).sum()) == 1


def test_a_width_of_more_blocks_than_any(wq, ctx):  # noqa: F811
    T, F, C = 2, 8192 * 2048 + 72, 8
    X, Wg, Wu = integers((T, C), 1, HALF), integers((F, C), 2, HALF), integers((F, C), 3, HALF)
    g, u, dH = integers((T, F), 5, HALF, 32, 64), integers((T, F), 6, HALF, -40, 41), torch.zeros((T, F), dtype=HALF, device="cuda")
    dH[1, -1], dH[0, 3] = 2, 1                     # few, so that the sums of dX stay exact
    got = wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=g, up=u)
    for t, f in ((1, F - 1), (0, 3)):
        dg, du = dH[t, f].double() * u[t, f].double(), dH[t, f].double() * g[t, f].double()
        assert torch.equal(got["dx"][t], (dg * Wg[f].double() + du * Wu[f].double()).half())
        assert torch.equal(got["dWg"][f], (dg * X[t].double()).half()) and torch.equal(got["dWu"][f], (du * X[t].double()).half())
    assert int((got["dWg"] != 0).any(dim=1).sum()) <= 2 and int((got["dWu"] != 0).any(dim=1).sum()) <= 2


def test_no_tokens(wq, ctx):  # noqa: F811
    X, Wg, Wu = block(4, 96, 64, HALF, 2)
    f = wq.windq_gated_forward(ctx, X[:0], Wg, Wu, want_saved=True)
    assert f["h"].shape == (0, 96)
    whole = torch.full((96, 72), 5.0, dtype=HALF, device="cuda")
    got = wq.windq_gated_backward(ctx, X[:0], Wg, Wu, f["h"], gate=f["gate"], up=f["up"],
                                  out=dict(dWg=whole[:, :64], dWu=torch.full((96, 72), 5.0, dtype=HALF, device="cuda")[:, :64]))
    assert got["dx"].shape == (0, 64) and bool((got["dWg"] == 0).all()) and bool((got["dWu"] == 0).all()) and bool((whole[:, 64:] == 5).all())


def test_weights_that_are_parts_of_one_matrix(wq, ctx):  # noqa: F811
    X, _, _ = block(50, 8, 128, BF, 1)
    both = integers((400, 128), 3, BF) / 16
    got = wq.windq_gated_forward(ctx, X, both[:200], both[200:])["h"]
    assert torch.equal(got, wq.windq_gated_forward(ctx, X, both[:200].clone(), both[200:].clone())["h"])


@pytest.mark.parametrize("dtype,act", [(HALF, "gelu"), (BF, "silu")])
@pytest.mark.parametrize("T,F,C", SIZES)
def test_int8_forward(wq, ctx, T, F, C, dtype, act):  # noqa: F811
    x, wg, wu = codes((T, C), 1), codes((F, C), 2), codes((F, C), 3)
    sx, sg, su = scales(T, 1), scales(F, 2) * 0.05, scales(F, 3)
    g, u = product(x, wg, sx, sg).double(), product(x, wu, sx, su).double()
    out, whole = padded(torch.zeros((T, F), dtype=dtype, device="cuda"), 8, 3.0)
    got = wq.windq_gated_int8_forward(ctx, padded(x, 16, 113)[0], sx, padded(wg, 16, 9)[0], sg, padded(wu, 16, -7)[0], su, activation=act,
                                      dtype=dtype, out=out)
    near(got, activation(g, act) * u, dtype)
    assert bool((whole[:, F:] == 3).all())


@pytest.mark.parametrize("T", [40, 700])
def test_graphs_and_streams(wq, T):  # noqa: F811
    """A training step captured once and replayed with other inputs, beside calls of another context on another stream."""
    F, C = 520, 264
    a, b = wq.windq_create(), wq.windq_create()
    X, Wg, Wu = block(T, F, C, HALF, 4)
    dH = integers((T, F), 8, HALF)

    def step(c, **k):
        f = wq.windq_gated_forward(c, X, Wg, Wu, want_saved=True, **k)
        return [f["h"], *wq.windq_gated_backward(c, X, Wg, Wu, dH, gate=f["gate"], up=f["up"], **k).values()]

    step(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(a)
    side = torch.cuda.Stream()
    for seed in (11, 12):
        X.copy_(integers((T, C), seed, HALF))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            other = step(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, other))
        assert all(torch.equal(p, q) for p, q in zip(out, step(a)))
    assert wq.windq_stalls(a) == 0 and wq.windq_stalls(b) == 0
    del graph
    torch.cuda.synchronize()
    wq.windq_destroy(a)
    wq.windq_destroy(b)


@pytest.mark.parametrize("T,F,C", [(30, 600, 4096), (100, 200, 8192)])
def test_reserved_scratch_is_enough_and_none_grows_while_captured(wq, T, F, C):  # noqa: F811
    X, Wg, Wu = block(T, F, C, HALF, 4)
    dH, c = integers((T, F), 8, HALF), wq.windq_create()
    x, w, sx, sw = codes((T, C), 1), codes((F, C), 2), scales(T, 1), scales(F, 2)
    want = wq.windq_gated_backward(c, X, Wg, Wu, dH)
    y = wq.windq_int8_forward(c, x, sx, w, sw)
    wq.windq_destroy(c)
    c = wq.windq_create()
    wq.windq_reserve(c, max(wq.windq_scratch_bytes_gated_backward(T, C, F, True), wq.windq_scratch_bytes_gated_forward(T, C, F),
                            wq.windq_scratch_bytes_int8_forward(T, F, C)))
    free = torch.cuda.mem_get_info()[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                                       # a cudaMalloc in here would end the capture
        got = wq.windq_gated_backward(c, X, Wg, Wu, dH)
        z = wq.windq_int8_forward(c, x, sx, w, sw)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want) and torch.equal(z, y)
    assert free - torch.cuda.mem_get_info()[0] < 64 << 20
    del graph
    torch.cuda.synchronize()
    wq.windq_destroy(c)


def test_refusals(wq, ctx):  # noqa: F811
    X, Wg, Wu = block(4, 96, 64, HALF, 2)
    dH = torch.zeros((4, 96), dtype=HALF, device="cuda")
    for wrong in ((X.float(), Wg, Wu), (X, Wg.to(BF), Wu), (X, Wg.cpu(), Wu)):
        with pytest.raises(TypeError):
            wq.windq_gated_forward(ctx, *wrong)
    for wrong in ((X, Wg[:, :56], Wu[:, :56]), (X, Wg[:90], Wu), (X.T, Wg, Wu), (X[0], Wg, Wu)):
        with pytest.raises(ValueError):
            wq.windq_gated_forward(ctx, *wrong)
    with pytest.raises(ValueError):
        wq.windq_gated_forward(ctx, X, Wg, Wu, activation="relu")
    with pytest.raises(ValueError):
        wq.windq_gated_backward(ctx, X, Wg, Wu, dH, gate=dH)
    with pytest.raises(ValueError):
        wq.windq_gated_backward(ctx, X, Wg, Wu, dH[:3])
    with pytest.raises(ValueError):
        wq.windq_gated_forward(ctx, X, Wg, Wu, want_saved=True, out=dict(gate=torch.empty((4, 104), dtype=HALF, device="cuda")[:, :96]))
    with pytest.raises(wq.WindqError) as e:
        wq.windq_gated_backward(ctx, X, Wg, Wu, dH, want_dx=False, want_dw=False)
    assert e.value.status == 1
    at = lambda t: t.data_ptr()  # noqa: E731
    forward = lambda T, C, ld, F: wq._lib.windq_gated_forward(ctx._h, 0, 0, at(X), T, C, ld, at(Wg), ld, at(Wu), ld, F, at(dH),  # noqa: E731
                                                              F + -F % 8, None, None, 0, None)
    assert forward(4, 1 << 26, 1 << 26, 96) == 2 and forward(4, 64, 64, 1 << 26) == 2 and forward((1 << 31) - 256, 64, 64, 96) == 2
    assert forward(-1, 64, 64, 96) == 2 and forward(4, 0, 64, 96) == 2 and forward(4, 65, 64, 96) == 2
    assert wq._lib.windq_gated_backward(ctx._h, 0, 0, at(X), 1 << 28, 64, 64, at(Wg), 64, at(Wu), 64, 96, None, None, 0, at(dH), 96, at(X), 64,
                                        None, None, 0, None) == 2
    odd = torch.zeros((4, 68), dtype=HALF, device="cuda")[:, :64]
    with pytest.raises(wq.WindqError) as e:
        wq.windq_gated_forward(ctx, odd, Wg, Wu)
    assert e.value.status == 3
    with pytest.raises(wq.WindqError) as e:
        wq.windq_gated_backward(ctx, X, Wg, Wu, torch.zeros((4, 97), dtype=HALF, device="cuda")[:, :96])
    assert e.value.status == 3
