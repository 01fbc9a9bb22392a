"""The context's scratch buffer: it grows under captured calls, and what it takes stays bounded."""
import pytest
import torch

from test_gpu_lora import HALF, backward, ctx, exact, forward, inputs, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_captured_call_outlives_the_growth_of_scratch(wq):  # noqa: F811
    own = wq.windq_create(0)
    try:
        q, dY = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=30)
        y, out = torch.zeros((24, 264), dtype=HALF, device="cuda"), {}
        forward(wq, own, q, out=y)
        out.update(backward(wq, own, q, dY))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            forward(wq, own, q, out=y)
            backward(wq, own, q, dY, out=out)
        wq.windq_reserve(own, 300 << 20)                       # several sizes, and a call that works in the new buffer
        big, big_dY = inputs(2600, 520, 1032, 64, 3, HALF, "segments", seed=31)
        backward(wq, own, big, big_dY)
        other = torch.full((64 << 20,), 0x55, dtype=torch.uint8, device="cuda")   # whoever gets freed memory writes to it
        for t in (y, *out.values()):
            t.zero_()
        new, new_dY = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=32)
        for k in q:
            q[k].copy_(new[k])
        dY.copy_(new_dY)
        graph.replay()
        torch.cuda.synchronize()
        want = exact(new, new_dY)
        assert torch.equal(y, want["y"].to(HALF)) and torch.equal(out["dx"], want["dx"].to(HALF))
        assert torch.equal(out["dA"], want["dA"].float()) and torch.equal(out["dB"], want["dB"].float())
        assert bool((other == 0x55).all())
        del graph
    finally:
        torch.cuda.synchronize()
        wq.windq_destroy(own)


def test_growing_step_by_step_takes_twice_the_last_buffer_at_most(wq):  # noqa: F811
    own = wq.windq_create(0)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    for mb in range(1, 65):
        wq.windq_reserve(own, mb << 20)
    taken = before - torch.cuda.mem_get_info()[0]
    # the last buffer is 64 to 127 MB, those before it half as much each; the driver hands out 2 MB at a time
    assert taken <= (2 * 127 + 2 * 8) << 20
    wq.windq_destroy(own)
    assert before - torch.cuda.mem_get_info()[0] <= 4 << 20
