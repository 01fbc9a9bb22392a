"""The adapter calls on two streams at once, each with a context of its own, as the ordering rule of the header asks."""
import pytest
import torch

from test_gpu_lora import BF, HALF, backward, ctx, exact, forward, inputs, wq  # noqa: F401

pytestmark = pytest.mark.gpu

# T, R, C, rank, adapters, kind: low-rank blocks of 64 to 256 columns of tensor memory in clusters of up to eight, beside
# tall tiles of 32 to 256 columns, split and not, and wide ones
ONE = [(48, 1032, 4104, 128, 48, "distinct"), (200, 2056, 2056, 128, 7, "mixed"), (700, 1288, 2056, 64, 3, "segments"), (96, 520, 1032, 72, 9, "mixed")]
TWO = [(16, 1032, 4104, 16, 16, "distinct"), (1, 2056, 2056, 8, 2, "one"), (255, 1288, 2056, 32, 31, "mixed"), (340, 200, 4104, 16, 3, "segments")]


def test_two_contexts_on_two_streams(wq):  # noqa: F811
    contexts = [wq.windq_create(0), wq.windq_create(0)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    try:
        jobs = [[inputs(*shape[:5], HALF if k else BF, shape[5], seed=20 + k) for shape in shapes] for k, shapes in enumerate((ONE, TWO))]
        for c in contexts:
            wq.windq_reserve(c, 8 << 20)
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        got = []
        for turn in range(12):
            for i in range(len(ONE)):
                for k in range(2):
                    q, dY = jobs[k][(i + turn * k) % len(ONE)]
                    with torch.cuda.stream(streams[k]):
                        got.append((k, (i + turn * k) % len(ONE), forward(wq, contexts[k], q), backward(wq, contexts[k], q, dY)))
        for s in streams:
            s.synchronize()
        want = [[exact(q, dY) for q, dY in j] for j in jobs]
        for k, i, y, back in got:
            w, dt = want[k][i], y.dtype
            assert torch.equal(y, w["y"].to(dt)) and torch.equal(back["dx"], w["dx"].to(dt)), (k, i)
            assert torch.equal(back["dA"], w["dA"].float()) and torch.equal(back["dB"], w["dB"].float()), (k, i)
        assert [wq.windq_stalls(c) for c in contexts] == [0, 0]
    finally:
        for c in contexts:
            wq.windq_destroy(c)
