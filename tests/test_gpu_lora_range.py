"""Low-rank values far below and far above fp16's own range, with an other factor that brings the result back into it: the
low-rank term keeps its precision on either type, token by token."""
import pytest
import torch

from test_gpu_lora import BF, HALF, SHAPES, backward, ctx, exact, forward, gen, ids_of, inputs, padded, wq  # noqa: F401

pytestmark = pytest.mark.gpu

POWERS = (-26, -13, 0, 13)
SOME = SHAPES[:16:2] + SHAPES[16::3] + [(240, 1096, 1096, 24, 7, "mixed"), (500, 9001, 520, 16, 3, "segments"), (700, 2600, 2056, 64, 3, "segments"),
                                        (2600, 4104, 1544, 32, 5, "segments")]


@pytest.mark.parametrize("T,R,C,r,n,kind", SOME)
def test_integers_times_powers_of_two_are_exact(wq, ctx, T, R, C, r, n, kind):  # noqa: F811
    """scaling[a] = 2^s and the other factor 2^(-11 - s): every sum is one of integers times 2^-11, or times 2^s in u, v, dA
    and dB, and exact.  fp16 alone keeps nothing of u below 2^-25 and nothing above 65504."""
    g = gen(T + 7)
    q, dY = inputs(T, R, C, r, n, HALF, kind, seed=50)
    s = torch.tensor(POWERS, device="cuda")[torch.randint(0, 4, (n,), generator=g, device="cuda")].float()
    q["scaling"] = torch.exp2(s)
    q["W"] = (q["W"].float() * 2.0 ** -11).to(HALF)
    for key in "BA":     # u is taken times B, v times A
        p = dict(q, **{key: (q[key].float() * torch.exp2(-11 - s)[:, None, None]).to(HALF)})
        want, got = exact(p, dY), backward(wq, ctx, p, dY)
        if key == "B":
            assert torch.equal(forward(wq, ctx, p), want["y"].to(HALF))
        else:
            assert torch.equal(got["dx"], want["dx"].to(HALF))
        assert torch.equal(got["dA"], want["dA"].float()) and torch.equal(got["dB"], want["dB"].float())


def low_rank_bound(q, z, left, right):
    """2^-16 of the token's largest low-rank value (16 bits at least) times the sum of |right|: [T, N]; left [n, r, K], right [n, N, r]."""
    out = torch.zeros((z.shape[0], right.shape[1]), dtype=torch.float64, device="cuda")
    for a in range(left.shape[0]):
        at = torch.nonzero(q["ids"] == a).flatten()
        top = (q["scaling"][a].double() * z[at].double() @ left[a].double().T).abs().amax(dim=1)
        out[at] = 2.0 ** -16 * top[:, None] * right[a].double().abs().sum(dim=1)[None, :]
    return out


@pytest.mark.parametrize("dt", [HALF, BF])
@pytest.mark.parametrize("scale", [2.0 ** -17, 2.0 ** -9, 2.0 ** 9])
@pytest.mark.parametrize("T,R,C,r,n,kind", [(1, 264, 520, 16, 1, "one"), (37, 264, 1032, 16, 5, "mixed"), (150, 1032, 2056, 64, 3, "segments"),
                                            (700, 520, 264, 128, 3, "mixed")])
def test_real_values_of_unequal_size(wq, ctx, T, R, C, r, n, kind, scale, dt):  # noqa: F811
    """Tokens and gradients of very unequal size; the other factor is large where they are small.  Beside the rounding of the
    result and that of two binary32 sums there is only that of the low-rank values."""
    q, dY = inputs(T, R, C, r, n, dt, kind, seed=51, integers=False)
    g = gen(T)
    size = torch.exp2(torch.randint(-4, 5, (T, 1), generator=g, device="cuda").float())
    q["X"], dY = (q["X"].float() * size * scale / C ** 0.5).to(dt), padded((dY.float() * size * scale / R ** 0.5).to(dt))
    q["W"] = (q["W"].float() * 2.0 ** -10).to(dt)
    big = min(8.0, 2.0 ** -6 / scale) if scale < 1 else 2.0 ** -8
    rounding, least = (2.0 ** -11, 2.0 ** -25) if dt == HALF else (2.0 ** -8, 0.0)
    p = dict(q, B=(q["B"].float() * big).to(dt))
    want = exact(p, dY)
    off = (forward(wq, ctx, p).double() - want["y"]).abs()
    assert bool((off <= rounding * want["y"].abs() + least + 2.0 ** -24 * (C + r + 8) * want["y_abs"] + low_rank_bound(p, p["X"], p["A"], p["B"])).all())
    p = dict(q, A=(q["A"].float() * big).to(dt))
    want = exact(p, dY)
    off = (backward(wq, ctx, p, dY, want_dab=False)["dx"].double() - want["dx"]).abs()
    bound = low_rank_bound(p, dY, p["B"].transpose(1, 2), p["A"].transpose(1, 2))
    assert bool((off <= rounding * want["dx"].abs() + least + 2.0 ** -24 * (R + r + 8) * want["dx_abs"] + bound).all())


def test_small_gradients_reach_dx(wq, ctx):  # noqa: F811
    # dY far below the normal range of fp16, as without loss scaling, and adapters of ordinary size
    q, dY = inputs(300, 264, 520, 16, 3, HALF, "mixed", seed=5, integers=False)
    dY = (dY.float() * 2.0 ** -20).to(HALF)
    q["W"] = torch.zeros_like(q["W"])
    q["B"] = (q["B"].float() / 16).to(HALF)
    want = exact(q, dY)
    off = (backward(wq, ctx, q, dY, want_dab=False)["dx"].double() - want["dx"]).abs()
    bound = low_rank_bound(q, dY, q["B"].transpose(1, 2), q["A"].transpose(1, 2))
    assert bool((off <= 2.0 ** -11 * want["dx"].abs() + 2.0 ** -25 + 2.0 ** -24 * (264 + 16 + 8) * want["dx_abs"] + bound).all())
