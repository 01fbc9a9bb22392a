"""New outputs of a call on a stream of the caller's do not lie in memory that the current stream still uses."""
import pytest
import torch

from test_gpu_quantize_rows import HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu

T, F, C = 1024, 2048, 1024      # every output takes a block of its own from the allocator


def calls(wq, c):
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    X, Wg, Wu, dH = r(T, C), 0.05 * r(F, C), 0.05 * r(F, C), r(T, F)
    x, a, b = (wq.windq_quantize_rows(c, t) for t in (X, Wg, Wu))
    f = wq.windq_gated_forward(c, X, Wg, Wu, want_saved=True)
    int8 = (x["codes"], x["scale"], a["codes"], a["scale"])
    return {"quantize_rows": lambda **k: wq.windq_quantize_rows(c, Wg, want_values=True, **k),
            "int8_forward": lambda **k: {"y": wq.windq_int8_forward(c, *int8, **k)},
            "gated_int8_forward": lambda **k: {"h": wq.windq_gated_int8_forward(c, *int8, b["codes"], b["scale"], **k)},
            "gated_forward": lambda **k: wq.windq_gated_forward(c, X, Wg, Wu, want_saved=True, **k),
            "gated_backward": lambda **k: wq.windq_gated_backward(c, X, Wg, Wu, dH, gate=f["gate"], up=f["up"], **k)}


@pytest.mark.parametrize("name", ["quantize_rows", "int8_forward", "gated_int8_forward", "gated_forward", "gated_backward"])
def test_memory_of_the_current_stream_is_left_alone(wq, ctx, name):  # noqa: F811
    call, side = calls(wq, ctx)[name], torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    used = [torch.empty(t.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda") for t in want.values()]
    torch.cuda._sleep(200_000_000)               # a tenth of a second in which the current stream has work left on them
    for t in used:
        t.fill_(255)
    del t, used
    got = call(stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_in_a_captured_side_stream(wq, ctx):  # noqa: F811
    call, side = calls(wq, ctx)["gated_forward"], torch.cuda.Stream()
    want = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        for t in got.values():
            t.zero_()
        graph.replay()
        assert all(torch.equal(got[k], want[k]) for k in want)
    del graph
    torch.cuda.synchronize()
