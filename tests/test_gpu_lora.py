"""The shared projection with low-rank adapters, and its gradients, against a plain implementation in 64 bits.

Most cases use small integers: every product and every sum is then exact in binary32, whatever its order, so that the
result must be the exact one rounded once to the output's type -- equal bits, no tolerance.  Cases with real values use a
bound derived from the number of roundings."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF, BF = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wq():
    import paper_2605_26660_b200 as wq
    return wq


@pytest.fixture(scope="module")
def ctx(wq):
    c = wq.windq_create(0)
    yield c
    wq.windq_destroy(c)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def padded(t):
    """The same rows at a stride that is a multiple of 8, as the calls want it (and return it)."""
    ld = t.shape[1] + -t.shape[1] % 8
    return torch.empty((t.shape[0], ld), dtype=t.dtype, device=t.device)[:, : t.shape[1]].copy_(t)


def ids_of(kind, T, n, g):
    if kind == "mixed":
        return torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "none":
        return torch.full((T,), -1, dtype=torch.int32, device="cuda")
    if kind == "one":
        return torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
    if kind == "distinct":
        return torch.arange(T, device="cuda", dtype=torch.int32) % n
    if kind == "invalid":       # indices no adapter has: such tokens have none
        ids = torch.randint(0, n, (T,), generator=g, device="cuda", dtype=torch.int32)
        ids[::3] = n
        ids[1::7] = -2147483648
        ids[2::11] = 2147483647
        return ids
    assert kind == "segments"   # runs of unequal length
    cut = torch.rand(T, generator=g, device="cuda") < 0.02
    return ((cut.cumsum(0) * 7 + 1) % (n + 1) - 1).to(torch.int32)


def inputs(T, R, C, r, n, dt, kind, seed=0, integers=True):
    g = gen(1000 * seed + T + R + C)
    if integers:
        small = lambda *s: (torch.randint(-1, 2, s, generator=g, device="cuda") * (torch.rand(s, generator=g, device="cuda") < 0.5))  # noqa: E731
        scaling = 2.0 ** torch.randint(-1, 2, (n,), generator=g, device="cuda").float()
    else:
        small = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        scaling = 0.5 + torch.rand(n, generator=g, device="cuda")
    q = dict(X=small(T, C), W=small(R, C), A=small(n, r, C), B=small(n, R, r))
    q = {k: v.to(dt) for k, v in q.items()}
    q["scaling"], q["ids"] = scaling, ids_of(kind, T, n, g)
    return q, padded(small(T, R).to(dt))


def exact(q, dY=None):
    """In 64 bits, adapter by adapter; the absolute sums beside them are what roundings are relative to."""
    x, w, a, b = (q[k].double() for k in "XWAB")
    s, ids = q["scaling"].double(), q["ids"]
    y, ya = x @ w.T, x.abs() @ w.abs().T
    out = dict(y=y, y_abs=ya)
    if dY is not None:
        dy = dY.double()
        out.update(dx=dy @ w, dx_abs=dy.abs() @ w.abs(), dA=torch.zeros_like(a), dB=torch.zeros_like(b),
                   dA_abs=torch.zeros_like(a), dB_abs=torch.zeros_like(b))
    for k in range(a.shape[0]):
        at = torch.nonzero(ids == k).flatten()
        u, ua = s[k] * x[at] @ a[k].T, s[k] * x[at].abs() @ a[k].abs().T
        y[at] += u @ b[k].T
        ya[at] += ua @ b[k].abs().T
        if dY is None:
            continue
        v, va = s[k] * dy[at] @ b[k], s[k] * dy[at].abs() @ b[k].abs()
        out["dx"][at] += v @ a[k]
        out["dx_abs"][at] += va @ a[k].abs()
        out["dA"][k], out["dB"][k] = v.T @ x[at], dy[at].T @ u
        out["dA_abs"][k], out["dB_abs"][k] = va.T @ x[at].abs(), dy[at].abs().T @ ua
    return out


def forward(wq, ctx, q, **kw):
    return wq.windq_lora_forward(ctx, q["X"], q["W"], q["A"], q["B"], q["scaling"], q["ids"], **kw)


def backward(wq, ctx, q, dY, **kw):
    return wq.windq_lora_backward(ctx, q["X"], q["W"], q["A"], q["B"], q["scaling"], q["ids"], dY, **kw)


SHAPES = [  # T, R, C, rank, adapters, kind
    (1, 8, 8, 8, 1, "one"), (1, 130, 72, 8, 3, "one"), (1, 257, 1032, 128, 2, "one"), (2, 1, 64, 16, 1, "mixed"),
    (3, 257, 40, 16, 2, "mixed"), (15, 64, 200, 24, 5, "mixed"), (16, 128, 64, 16, 16, "distinct"), (17, 300, 328, 40, 5, "mixed"),
    (31, 129, 512, 64, 7, "invalid"), (33, 1000, 264, 8, 33, "distinct"), (48, 520, 136, 16, 32, "mixed"), (64, 72, 1000, 56, 4, "segments"),
    (65, 384, 96, 128, 3, "mixed"), (100, 256, 256, 32, 100, "distinct"), (128, 264, 392, 16, 9, "mixed"), (129, 136, 512, 40, 3, "none"),
    (200, 264, 72, 72, 6, "mixed"), (255, 513, 128, 8, 2, "segments"), (256, 248, 456, 16, 64, "distinct"), (257, 96, 640, 24, 3, "mixed"),
    (300, 520, 648, 64, 40, "mixed"), (511, 40, 88, 16, 2, "segments"), (640, 777, 320, 120, 5, "segments"), (1025, 512, 1032, 16, 4, "invalid"),
    (2100, 264, 520, 32, 3, "segments"), (48, 640, 4160, 16, 24, "mixed"), (203, 1200, 8192, 32, 48, "mixed"), (330, 520, 6000, 16, 30, "mixed"),
    # tiles that are split along the reduction, at every height of a tile whose sums share its memory
    (112, 200, 1096, 16, 3, "mixed"), (144, 1030, 2056, 48, 3, "segments"), (192, 2056, 1032, 8, 20, "mixed"), (208, 136, 4104, 32, 3, "mixed"),
    (209, 2050, 2056, 64, 3, "segments"), (240, 1096, 1096, 24, 7, "mixed"), (256, 4104, 4104, 16, 5, "segments"), (258, 4100, 4104, 128, 3, "mixed"),
    (300, 1096, 2056, 24, 5, "mixed"), (320, 264, 1096, 16, 2, "segments"),
    # wide tiles: few and many, split along the reduction or not, of odd widths
    (321, 200, 8200, 16, 3, "segments"), (700, 2600, 2056, 64, 3, "segments"), (777, 5120, 1032, 8, 6, "segments"), (1300, 3000, 1096, 40, 4, "mixed"),
    (500, 9001, 520, 16, 3, "segments"), (2600, 4104, 1544, 32, 5, "segments"), (4100, 700, 4104, 16, 2, "segments"), (350, 40, 130 * 64, 8, 1, "one"), (3000, 1288, 136, 8, 1, "one"),
]


@pytest.mark.parametrize("dt", [HALF, BF])
@pytest.mark.parametrize("T,R,C,r,n,kind", SHAPES)
def test_integers_are_exact(wq, ctx, T, R, C, r, n, kind, dt):
    q, dY = inputs(T, R, C, r, n, dt, kind)
    want = exact(q, dY)
    got = forward(wq, ctx, q)
    assert got.shape == (T, R) and torch.equal(got, want["y"].to(dt))
    back = backward(wq, ctx, q, dY)
    assert torch.equal(back["dx"], want["dx"].to(dt))
    assert torch.equal(back["dA"], want["dA"].float()) and torch.equal(back["dB"], want["dB"].float())


@pytest.mark.parametrize("dt", [HALF, BF])
@pytest.mark.parametrize("T,R,C,r,n,kind", SHAPES[1::3] + [(96, 512, 2048, 8, 1, "one"), (40, 2048, 4096, 16, 8, "mixed"),
                                                          (700, 640, 2056, 32, 3, "segments")])
def test_real_values(wq, ctx, T, R, C, r, n, kind, dt):
    """u = 2^-24: a sum of K products is off by at most K u times the sum of their absolute values; a low-rank term goes
    through two such sums and one rounding to 22 (fp16 pairs) or 16 (bf16 pairs) bits."""
    q, dY = inputs(T, R, C, r, n, dt, kind, seed=2, integers=False)
    want, u = exact(q, dY), 2.0 ** -24
    rounding = 2.0 ** -11 if dt == HALF else 2.0 ** -8
    pair = 2.0 ** -21 if dt == HALF else 2.0 ** -16
    y = forward(wq, ctx, q).double()
    assert bool(((y - want["y"]).abs() <= rounding * want["y"].abs() + (u * (C + r + 8) + pair) * want["y_abs"] + 1e-7).all())
    back = backward(wq, ctx, q, dY)
    assert bool(((back["dx"].double() - want["dx"]).abs()
                 <= rounding * want["dx"].abs() + (u * (R + r + 8) + pair) * want["dx_abs"] + 1e-7).all())
    for k, K in (("dA", R), ("dB", C)):
        assert bool(((back[k].double() - want[k]).abs() <= u * (K + T + 16) * want[k + "_abs"]).all()), k
        norm = float((back[k].double() - want[k]).norm() / want[k].norm().clamp_min(1e-30))
        assert norm <= 1e-5, (k, norm)   # roundings are not all of one sign: binary32 results, not 16-bit ones


def test_small_and_large_gradients_keep_32_bits(wq, ctx):
    # dY far below and far above the normal range of fp16: dA and dB are binary32 sums of products of fp16 values
    for scale in (2.0 ** -20, 2.0 ** 10):
        q, dY = inputs(300, 264, 520, 16, 3, HALF, "mixed", seed=5, integers=False)
        dY = (dY.float() * scale).to(HALF)
        want, back = exact(q, dY), backward(wq, ctx, q, dY)
        for k in ("dA", "dB"):
            assert float((back[k].double() - want[k]).norm() / want[k].norm()) <= 1e-5, (k, scale)


@pytest.mark.parametrize("T", [1, 5, 70, 300])
def test_strides_and_outputs_of_the_caller(wq, ctx, T):
    R, C, r, n = 203, 264, 24, 4
    q, dY = inputs(T, R, C, r, n, HALF, "mixed", seed=3)
    want = exact(q, dY)
    wide = lambda t, ld: torch.full((t.shape[0] + 1, ld), 3.0, dtype=t.dtype, device="cuda")  # noqa: E731
    X, W, D = wide(q["X"], 296), wide(q["W"], 320), wide(dY, 216)
    X[:T, 8: 8 + C], W[:R, 16: 16 + C], D[:T, :R] = q["X"], q["W"], dY
    p = dict(q, X=X[:T, 8: 8 + C], W=W[:R, 16: 16 + C])
    Y, dX = torch.full((T + 1, 240), 9.0, dtype=HALF, device="cuda"), torch.full((T + 1, 288), 9.0, dtype=HALF, device="cuda")
    forward(wq, ctx, p, out=Y[:T, :R])
    assert torch.equal(Y[:T, :R], want["y"].to(HALF)) and bool((Y[T] == 9).all()) and bool((Y[:, R:] == 9).all())
    out = dict(dx=dX[:T, :C], dA=torch.full((n, r, C), 5.0, device="cuda"), dB=torch.full((n, R, r), 5.0, device="cuda"))
    back = backward(wq, ctx, p, D[:T, :R], out=out)
    assert back["dA"] is out["dA"] and back["dB"] is out["dB"]
    assert torch.equal(dX[:T, :C], want["dx"].to(HALF)) and bool((dX[T] == 9).all()) and bool((dX[:, C:] == 9).all())
    assert torch.equal(out["dA"], want["dA"].float()) and torch.equal(out["dB"], want["dB"].float())


def test_parts_of_the_gradient(wq, ctx):
    q, dY = inputs(150, 136, 264, 16, 3, BF, "mixed", seed=4)
    want = exact(q, dY)
    a = backward(wq, ctx, q, dY, want_dab=False)
    b = backward(wq, ctx, q, dY, want_dx=False)
    assert a["dA"] is None and a["dB"] is None and b["dx"] is None
    assert torch.equal(a["dx"], want["dx"].to(BF))
    assert torch.equal(b["dA"], want["dA"].float()) and torch.equal(b["dB"], want["dB"].float())


def test_gradients_against_differences(wq, ctx):
    # Y is linear in A, in B and in X: on integers the central difference of sum(dY * Y) is the exact derivative
    T, R, C, r, n = 150, 136, 264, 16, 3
    q, dY = inputs(T, R, C, r, n, HALF, "mixed", seed=6)
    q["scaling"].fill_(1.0)
    back = backward(wq, ctx, q, dY)
    g = gen(77)
    for key, grad in (("A", back["dA"]), ("B", back["dB"]), ("X", back["dx"])):
        E = torch.randint(-1, 2, q[key].shape, generator=g, device="cuda").to(HALF)
        E *= torch.rand(E.shape, generator=g, device="cuda") < 0.1
        loss = lambda sign: float((dY.double() * forward(wq, ctx, dict(q, **{key: q[key] + sign * E})).double()).sum())  # noqa: E731
        assert (loss(1) - loss(-1)) / 2 == float((grad.double() * E.double()).sum()), key


def test_a_token_that_is_not_finite_stays_alone(wq, ctx):
    T, R, C, r, n = 200, 136, 264, 16, 4
    q, dY = inputs(T, R, C, r, n, HALF, "segments", seed=8)
    q["ids"] = (torch.arange(T, device="cuda") // 50).to(torch.int32)
    want = exact(q, dY)
    q["X"][7, 3], q["X"][8, 5] = float("nan"), float("inf")
    dY[9, 2] = float("-inf")
    y, back = forward(wq, ctx, q), backward(wq, ctx, q, dY)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[7] = rest[8] = False
    assert torch.equal(y[rest], want["y"].to(HALF)[rest])
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[9] = False
    assert torch.equal(back["dx"][rest], want["dx"].to(HALF)[rest])
    assert torch.equal(back["dA"][1:], want["dA"].float()[1:]) and torch.equal(back["dB"][1:], want["dB"].float()[1:])


def test_no_tokens(wq, ctx):
    q, dY = inputs(5, 136, 264, 16, 3, HALF, "mixed")
    q["X"], q["ids"], dY = q["X"][:0], q["ids"][:0], dY[:0]
    assert forward(wq, ctx, q).shape == (0, 136)
    back = backward(wq, ctx, q, dY)
    assert back["dx"].shape == (0, 264) and not back["dA"].any() and not back["dB"].any()


@pytest.mark.parametrize("T", [3, 90, 700])
def test_equal_calls_give_equal_bits(wq, ctx, T):
    q, dY = inputs(T, 520, 1032, 16, 5, HALF, "mixed", seed=9, integers=False)
    y, back = forward(wq, ctx, q), backward(wq, ctx, q, dY)
    for _ in range(3):
        assert torch.equal(forward(wq, ctx, q), y)
        again = backward(wq, ctx, q, dY)
        assert all(torch.equal(again[k], back[k]) for k in ("dx", "dA", "dB"))


def test_calls_of_different_sizes_in_a_row_on_a_side_stream(wq, ctx):
    side = torch.cuda.Stream()
    jobs = [inputs(T, R, C, r, n, HALF, "mixed", seed=10) for T, R, C, r, n in
            ((700, 264, 520, 32, 3), (1, 520, 264, 8, 2), (300, 136, 1032, 128, 4), (40, 264, 72, 16, 9))]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ys = [forward(wq, ctx, q) for q, _ in jobs]
        backs = [backward(wq, ctx, q, dY) for q, dY in jobs]
    side.synchronize()
    for (q, dY), y, back in zip(jobs, ys, backs):
        want = exact(q, dY)
        assert torch.equal(y, want["y"].to(HALF)) and torch.equal(back["dx"], want["dx"].to(HALF))
        assert torch.equal(back["dA"], want["dA"].float()) and torch.equal(back["dB"], want["dB"].float())


def test_a_captured_graph_replays(wq, ctx):
    q, _ = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=11)
    out = torch.empty((24, 264), dtype=HALF, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward(wq, ctx, q, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward(wq, ctx, q, out=out)
    other, _ = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=12)
    for k in q:
        q[k].copy_(other[k])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, exact(other)["y"].to(HALF))
    del graph


def test_refusals(wq, ctx):
    q, dY = inputs(8, 64, 64, 16, 3, HALF, "mixed")
    out = torch.full((8, 64), 7.0, dtype=HALF, device="cuda")
    half, cut = lambda t: t.to(BF), lambda t: t[:, :, :12].contiguous()  # noqa: E731
    for change, error in ((dict(W=half(q["W"])), TypeError), (dict(X=q["X"].float()), TypeError), (dict(ids=q["ids"].long()), TypeError),
                          (dict(A=q["A"].cpu()), TypeError), (dict(scaling=q["scaling"][:2]), ValueError), (dict(ids=q["ids"][:7]), ValueError),
                          (dict(X=q["X"][:, :56]), ValueError), (dict(W=q["W"].T), ValueError)):
        with pytest.raises(error):
            forward(wq, ctx, dict(q, **change), out=out)
    flat = torch.zeros(8 * 64 + 8, dtype=HALF, device="cuda")
    for change, status in ((dict(A=q["A"][:, :12].contiguous(), B=cut(q["B"])), 4),                    # rank 12
                           (dict(X=flat[1: 1 + 8 * 64].view(8, 64)), 3),                               # alignment
                           (dict(X=q["X"][:, :60], W=q["W"][:, :60], A=q["A"][:, :, :60].contiguous()), 2)):   # C % 8
        with pytest.raises(wq.WindqError) as e:
            forward(wq, ctx, dict(q, **change), out=out)
        assert e.value.status == status
    with pytest.raises(ValueError):
        forward(wq, ctx, q, out=out[:, :56])
    with pytest.raises(ValueError):
        backward(wq, ctx, q, dY[:7])
    with pytest.raises(wq.WindqError) as e:
        backward(wq, ctx, q, dY, want_dx=False, want_dab=False)
    assert e.value.status == 1
    torch.cuda.synchronize()
    assert bool((out == 7).all())


def test_no_wait_gave_up(wq, ctx):
    assert wq.windq_stalls(ctx) == 0
