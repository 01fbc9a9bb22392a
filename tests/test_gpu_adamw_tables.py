"""AdamW over more tensors than one launch takes: every result of every tensor, bit for bit, over two steps that nothing
waits between; and the step in a captured graph."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import B1, B2, EPS, LR, TORCH, WD, build, ctx, decode, encode_m, encode_r, f32, host, numpy_step, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [("f32", "f32", "bf16"), ("f16", "bf16", "bf16"), ("bf16", "f16", "f16")])
@pytest.mark.parametrize("count", [56, 57, 500])
def test_every_tensor_of_several_launches(wq, ctx, count, param, grad, copy, state):  # noqa: F811
    sizes = [0 if j % 61 == 60 else 1 + (173 * j) % 1500 for j in range(count)]
    P, G, M, V, kw, K, tensors = build(wq, sizes, param, grad, state, copy, seed=20)
    p, g = [host(x) for x in P], [host(x) for x in G]
    m, v = [np.zeros(n, f32) for n in sizes], [np.zeros(n, f32) for n in sizes]
    for t in (1, 2):
        wq.windq_adamw_step(ctx, tensors, step=t, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    values = wq.windq_adamw_states(ctx, tensors) if state == 8 else (M, V)
    torch.cuda.synchronize()
    for j, n in enumerate(sizes):
        codes = scales = None
        for t in (1, 2):
            new, m[j], v[j], r = numpy_step(p[j], g[j], m[j], v[j], t, 1.0)
            p[j] = torch.from_numpy(new).to(TORCH[param]).float().numpy()
            if state == 8:
                (qm, sm), (qr, sr) = encode_m(m[j]), encode_r(r)
                codes, scales = (qm, qr), (sm, sr)
                m[j], r = decode(qm, sm, 127), decode(qr, sr, 255)
                v[j] = r * r
        assert np.array_equal(host(P[j]), p[j]), j
        # rounded from the step's binary32 value, not from the 16-bit parameter
        assert torch.equal(K[j].cpu(), torch.from_numpy(new).to(TORCH[copy])), j
        assert np.array_equal(host(values[0][j]), m[j]) and np.array_equal(host(values[1][j]), v[j]), j
        if state == 8 and n:
            assert np.array_equal(M[j].cpu().numpy(), codes[0]) and np.array_equal(V[j].cpu().numpy(), codes[1]), j
            assert np.array_equal(host(kw["m_scale"][j]), scales[0]) and np.array_equal(host(kw["r_scale"][j]), scales[1]), j


@pytest.mark.parametrize("state", [32, 8])
def test_a_captured_step_repeats(wq, ctx, state):  # noqa: F811
    # the step number is the host's: a replay takes the step that was captured
    sizes = [700] * 80
    P, G, M, V, kw, K, tensors = build(wq, sizes, "f32", "f32", state, None, seed=21)
    first = [x.clone() for x in P]
    go = lambda ts: wq.windq_adamw_step(ctx, ts, step=7, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(tensors)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    P2, G2, M2, V2, kw2, _, again = build(wq, sizes, "f32", "f32", state, None, seed=21)
    assert all(torch.equal(a, b) for a, b in zip(first, P2))
    for _ in range(3):
        go(again)
    torch.cuda.synchronize()
    for a, b in ((P, P2), (M, M2), (V, V2), (kw.get("m_scale", []), kw2.get("m_scale", [])), (kw.get("r_scale", []), kw2.get("r_scale", []))):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    del graph
