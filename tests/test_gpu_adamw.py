"""AdamW over many tensors against a plain implementation.  The 32-bit arithmetic is a fixed sequence of IEEE operations,
so numpy repeats it bit for bit (codes and scales of 8-bit states included); against the formula in 64 bits the result is
off by the rounding of a handful of binary32 operations."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, WD = 3e-3, 0.9, 0.99, 1e-8, 0.05
f32 = np.float32


@pytest.fixture(scope="module")
def wq():
    import paper_2605_26660_b200 as wq
    return wq


@pytest.fixture(scope="module")
def ctx(wq):
    c = wq.windq_create(0)
    yield c
    wq.windq_destroy(c)


def blocks(x):
    pad = -len(x) % 256
    return np.concatenate([x, np.zeros(pad, x.dtype)]).reshape(-1, 256)


def encode(x, levels):
    a = np.abs(blocks(x))
    top = a.max(axis=1)
    top = np.where(top >= f32(2.0 ** -100), top, f32(0))
    inv = np.where(top > 0, f32(1) / np.where(top > 0, top, f32(1)), f32(0)).astype(f32)
    q = np.minimum(np.rint(np.sqrt(a * inv[:, None]) * f32(levels)), f32(levels))
    return q, top, a


def encode_m(m):
    q, top, _ = encode(m, 127)
    return (q * np.sign(blocks(m))).reshape(-1)[: len(m)].astype(np.int8), top


def encode_r(r):
    q, top, a = encode(r, 255)
    q = np.where((a > 0) & (top > 0)[:, None], np.maximum(q, f32(1)), q)
    return q.reshape(-1)[: len(r)].astype(np.uint8), top


def decode(q, scale, levels):
    u = q.astype(f32) * f32(1.0 / levels)
    return ((u * np.abs(u)) * np.repeat(scale, 256)[: len(q)]).astype(f32)


def numpy_step(p, g, m, v, t, gs):
    """p, g fp32; returns p, m, v, r in the order of operations of the header."""
    g = g * f32(gs)
    m = m * f32(B1) + g * f32(1.0 - B1)
    v = v * f32(B2) + (g * g) * f32(1.0 - B2)
    r = np.sqrt(v)
    p = p * f32(1.0 - LR * WD) - (m * f32(LR / (1.0 - B1 ** t))) / (r * f32(1.0 / math.sqrt(1.0 - B2 ** t)) + f32(EPS))
    return p, m, v, r


def exact_step(p, g, m, v, t, gs):
    g = g.astype(np.float64) * gs
    m = B1 * m.astype(np.float64) + (1 - B1) * g
    v = B2 * v.astype(np.float64) + (1 - B2) * g * g
    return (1 - LR * WD) * p.astype(np.float64) - LR * (m / (1 - B1 ** t)) / (np.sqrt(v / (1 - B2 ** t)) + EPS), m, v


SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 10001, 0, 3]
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.float().cpu().numpy()


def build(wq, sizes, param, grad, state, copy, seed=1, zero_grad=()):
    rng = np.random.default_rng(seed)
    cuda = lambda x, dt: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(dt)  # noqa: E731
    P = [cuda(rng.standard_normal(n).astype(f32), TORCH[param]) for n in sizes]
    G = [cuda((rng.standard_normal(n) * 10.0 ** rng.uniform(-6, 1)).astype(f32) * (j not in zero_grad), TORCH[grad])
         for j, n in enumerate(sizes)]
    bits8 = state == 8
    M = [torch.zeros(n, dtype=torch.int8 if bits8 else torch.float32, device="cuda") for n in sizes]
    V = [torch.zeros(n, dtype=torch.uint8 if bits8 else torch.float32, device="cuda") for n in sizes]
    scale = lambda: [torch.zeros(-(-n // 256), dtype=torch.float32, device="cuda") for n in sizes]  # noqa: E731
    kw = dict(m_scale=scale(), r_scale=scale()) if bits8 else {}
    K = None if copy is None else [torch.full((n,), -7.0, dtype=TORCH[copy], device="cuda") for n in sizes]
    return P, G, M, V, kw, K, wq.AdamwTensors(P, G, M, V, copies=K, **kw)


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [("f32", "f32", "f16"), ("f32", "bf16", "bf16"), ("f32", "f16", None),
                                             ("f16", "f16", None), ("bf16", "f32", None)])
def test_steps_repeat_the_operations_bit_for_bit(wq, ctx, state, param, grad, copy):
    P, G, M, V, kw, K, tensors = build(wq, SIZES, param, grad, state, copy, zero_grad=(4,))
    gs = torch.tensor([0.625], dtype=torch.float32, device="cuda")
    p = [host(x) for x in P]
    m, v = [np.zeros(n, f32) for n in SIZES], [np.zeros(n, f32) for n in SIZES]
    for t in (1, 2, 3, 1000):
        wq.windq_adamw_step(ctx, tensors, step=t, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD, grad_scale=gs)
        torch.cuda.synchronize()
        values = wq.windq_adamw_states(ctx, tensors) if state == 8 else (M, V)
        for j, n in enumerate(SIZES):
            if n == 0:
                continue
            g = host(G[j])
            ep, em, ev = exact_step(p[j], g, m[j], v[j], t, 0.625)
            new, nm, nv, nr = numpy_step(p[j], g, m[j], v[j], t, 0.625)
            # against 64 bits, u = 2^-24: p (1 - lr wd) is three roundings off; the update 16 at most (m 4, its factor and
            # product 3, sqrt(v) 3, its factor, product and sum 4, the quotient 1; m adds values of one sign here)
            update = np.abs(ep - (1 - LR * WD) * p[j].astype(np.float64))
            assert np.all(np.abs(new - ep) <= 2.0 ** -24 * (4 * np.abs(p[j]) + 17 * update))
            want = torch.from_numpy(new).to(TORCH[param])
            assert torch.equal(P[j].cpu(), want), ("param", t, n)
            if K is not None:
                assert torch.equal(K[j].cpu(), torch.from_numpy(new).to(TORCH[copy])), ("copy", t, n)
            p[j] = want.float().numpy()
            if state == 32:
                assert np.array_equal(host(M[j]), nm) and np.array_equal(host(V[j]), nv), ("states", t, n)
                m[j], v[j] = nm, nv
                continue
            (qm, sm), (qr, sr) = encode_m(nm), encode_r(nr)
            assert np.array_equal(M[j].cpu().numpy(), qm) and np.array_equal(V[j].cpu().numpy(), qr), ("codes", t, n)
            assert np.array_equal(host(kw["m_scale"][j]), sm) and np.array_equal(host(kw["r_scale"][j]), sr), ("scales", t, n)
            m[j] = decode(qm, sm, 127)
            r = decode(qr, sr, 255)
            v[j] = r * r
            assert np.array_equal(host(values[0][j]), m[j]) and np.array_equal(host(values[1][j]), v[j]), ("values", t, n)


def test_8_bit_states_follow_32_bit_ones(wq, ctx):
    # an element of at least half the block's largest has a code q >= 90 for m and >= 180 for r, so a rounding moves m by
    # 1/90 and r by 1/180 of itself at most; m carries 0.9 and v 0.99 of that on.  Over eight steps of one gradient the
    # worst case is 6.4 % for m and 4.3 % for r, 11 % for an update
    n = 4096
    rng = np.random.default_rng(3)
    g = rng.choice([-1.0, 1.0], n) * rng.uniform(0.5, 1.0, n)
    out = []
    for state in (32, 8):
        P, G, M, V, kw, K, tensors = build(wq, [n], "f32", "f32", state, None)
        P[0].zero_()
        G[0].copy_(torch.from_numpy(g.astype(f32)))
        for t in range(1, 9):
            wq.windq_adamw_step(ctx, tensors, step=t, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.0)
        out.append(host(P[0]))
    assert np.max(np.abs(out[0] - out[1])) <= 0.11 * np.max(np.abs(out[0]))


def test_tiny_and_empty_blocks(wq, ctx):
    # a zero gradient leaves an empty block empty; values below 2^-100 are dropped; neither divides by zero
    P, G, M, V, kw, K, tensors = build(wq, [512], "f32", "f32", 8, None, zero_grad=(0,))
    before = host(P[0])
    G[0][256:] = 1e-33
    wq.windq_adamw_step(ctx, tensors, step=1, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    torch.cuda.synchronize()
    assert not M[0].any() and not V[0].any() and not kw["m_scale"][0].any() and not kw["r_scale"][0].any()
    assert np.array_equal(host(P[0])[:256], before[:256] * f32(1 - LR * WD))
    assert np.isfinite(host(P[0])).all()


def test_many_tensors_take_several_tables(wq, ctx):
    sizes = [1 + (37 * j) % 600 for j in range(1000)]
    P, G, M, V, kw, K, tensors = build(wq, sizes, "f32", "f32", 32, "bf16")
    p = [host(x) for x in P]
    wq.windq_adamw_step(ctx, tensors, step=1, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    torch.cuda.synchronize()
    for j, n in enumerate(sizes):
        want = numpy_step(p[j], host(G[j]), np.zeros(n, f32), np.zeros(n, f32), 1, 1.0)[0]
        assert np.array_equal(host(P[j]), want), j


def test_other_gradients_and_a_side_stream(wq, ctx):
    P, G, M, V, kw, K, tensors = build(wq, [300, 4097], "f32", "f32", 32, None)
    p = [host(x) for x in P]
    H = [torch.randn_like(g) for g in G]
    tensors.set_grads(H)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wq.windq_adamw_step(ctx, tensors, step=1, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD, stream=side)
    side.synchronize()
    for j in range(2):
        n = len(p[j])
        assert np.array_equal(host(P[j]), numpy_step(p[j], host(H[j]), np.zeros(n, f32), np.zeros(n, f32), 1, 1.0)[0])


def test_refusals(wq, ctx):
    P, G, M, V, kw, K, tensors = build(wq, [64], "f32", "f32", 8, None)
    go = lambda **k: wq.windq_adamw_step(ctx, tensors, **{**dict(step=1, lr=LR), **k})  # noqa: E731
    for bad, status in ((dict(step=0), 4), (dict(lr=-1.0), 4), (dict(lr=float("nan")), 4), (dict(beta1=1.0), 4), (dict(beta2=-0.1), 4),
                        (dict(eps=0.0), 4), (dict(weight_decay=-1.0), 4)):
        with pytest.raises(wq.WindqError) as e:
            go(**bad)
        assert e.value.status == status, bad
    with pytest.raises(ValueError):
        wq.AdamwTensors(P, G, M, V)                                        # no scales
    with pytest.raises(ValueError):
        wq.AdamwTensors(P, [torch.zeros(63, device="cuda")], M, V, **kw)
    with pytest.raises(TypeError):
        wq.AdamwTensors(P, G, M, M, **kw)                                  # sqrt(v) codes are unsigned
    with pytest.raises(TypeError):
        wq.AdamwTensors([p.cpu() for p in P], G, M, V, **kw)
    big = torch.zeros(80, device="cuda")
    odd = wq.AdamwTensors([big[1:65]], G, M, V, **kw)                      # not 16-byte aligned
    before = M[0].clone()
    with pytest.raises(wq.WindqError) as e:
        wq.windq_adamw_step(ctx, odd, step=1, lr=LR)
    assert e.value.status == 3
    torch.cuda.synchronize()
    assert torch.equal(M[0], before) and not big.any()
    P32, G32, M32, V32, _, _, t32 = build(wq, [64], "f32", "f32", 32, None)
    with pytest.raises(ValueError):
        wq.windq_adamw_states(ctx, t32)
