"""A gradient that is not finite, or whose square overflows, in the AdamW step: what it does stays with its element."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import B1, B2, EPS, LR, WD, build, ctx, decode, encode_m, encode_r, f32, host, numpy_step, wq  # noqa: F401

pytestmark = pytest.mark.gpu

BAD = {3: np.nan, 5: np.inf, 6: -np.inf, 255: np.float32(1e30), 256: np.float32(-3e19), 600: np.nan, 700: np.float32(2e38)}
N = 701     # blocks of 256, 256 and 189 elements


@pytest.mark.parametrize("state", [8, 32])
def test_other_elements_keep_their_bits(wq, ctx, state):  # noqa: F811
    rng = np.random.default_rng(9)
    P, G, M, V, kw, K, tensors = build(wq, [N], "f32", "f32", state, "bf16", seed=9)
    p, m, v = host(P[0]), np.zeros(N, f32), np.zeros(N, f32)
    for t in (1, 2, 3, 4):
        g = (rng.standard_normal(N) * 0.01).astype(f32)
        if t == 2:
            for i, x in BAD.items():
                g[i] = x
        G[0].copy_(torch.from_numpy(g))
        wq.windq_adamw_step(ctx, tensors, step=t, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
        torch.cuda.synchronize()
        with np.errstate(all="ignore"):
            p, m, v, r = numpy_step(p, g, m, v, t, 1.0)
        assert np.array_equal(host(P[0]), p, equal_nan=True), t
        assert np.array_equal(host(K[0]), torch.from_numpy(p).bfloat16().float().numpy(), equal_nan=True), t
        if state == 32:
            assert np.array_equal(host(M[0]), m, equal_nan=True) and np.array_equal(host(V[0]), v, equal_nan=True), t
            continue
        fine = np.isfinite(r)
        assert t != 2 or set(np.flatnonzero(~fine)) == set(BAD)
        m, r = np.where(fine, m, f32(0)), np.where(fine, r, f32(0))
        (qm, sm), (qr, sr) = encode_m(m), encode_r(r)
        assert np.array_equal(M[0].cpu().numpy(), qm) and np.array_equal(V[0].cpu().numpy(), qr), t
        assert np.array_equal(host(kw["m_scale"][0]), sm) and np.array_equal(host(kw["r_scale"][0]), sr), t
        assert np.isfinite(sm).all() and np.isfinite(sr).all()
        m, r = decode(qm, sm, 127), decode(qr, sr, 255)
        v = r * r
        values = wq.windq_adamw_states(ctx, tensors)
        assert np.array_equal(host(values[0][0]), m) and np.array_equal(host(values[1][0]), v), t
    spoilt = [i for i, x in BAD.items() if not np.isfinite(x)]
    assert set(np.flatnonzero(~np.isfinite(p))) == set(spoilt)      # as the formula has it


def test_a_block_of_nothing_else(wq, ctx):  # noqa: F811
    P, G, M, V, kw, K, tensors = build(wq, [300], "f32", "f16", 8, None, seed=10)
    G[0].fill_(float("inf"))
    wq.windq_adamw_step(ctx, tensors, step=1, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    torch.cuda.synchronize()
    assert not M[0].any() and not V[0].any() and not kw["m_scale"][0].any() and not kw["r_scale"][0].any()
