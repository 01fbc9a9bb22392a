"""Python threads go on while a feed-forward call waits for room in its stream's queue."""
import threading
import time

import pytest
import torch

from test_gpu_quantize_rows import HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(wq, c):
    X, W = torch.ones((2, 64), dtype=HALF, device="cuda"), torch.ones((8, 64), dtype=HALF, device="cuda")
    x, w = wq.windq_quantize_rows(c, X), wq.windq_quantize_rows(c, W)
    y, f = torch.empty((2, 8), dtype=HALF, device="cuda"), wq.windq_gated_forward(c, X, W, W, want_saved=True)
    d = wq.windq_gated_backward(c, X, W, W, f["h"], gate=f["gate"], up=f["up"])
    return {"quantize_rows": lambda: wq.windq_quantize_rows(c, X, out=x),
            "int8_forward": lambda: wq.windq_int8_forward(c, x["codes"], x["scale"], w["codes"], w["scale"], out=y),
            "gated_int8_forward": lambda: wq.windq_gated_int8_forward(c, x["codes"], x["scale"], w["codes"], w["scale"], w["codes"], w["scale"], out=y),
            "gated_forward": lambda: wq.windq_gated_forward(c, X, W, W, out=f),
            "gated_backward": lambda: wq.windq_gated_backward(c, X, W, W, f["h"], gate=f["gate"], up=f["up"], out=d)}


@pytest.mark.parametrize("name", ["quantize_rows", "int8_forward", "gated_int8_forward", "gated_forward", "gated_backward"])
def test_other_threads_run_while_a_call_waits(wq, ctx, name):  # noqa: F811
    call, done, gaps = calls(wq, ctx)[name], threading.Event(), [0.0]

    def beat():
        last = time.perf_counter()
        while not done.is_set():
            time.sleep(0.002)
            now = time.perf_counter()
            gaps.append(now - last)
            last = now

    call()
    torch.cuda.synchronize()
    other = threading.Thread(target=beat)
    other.start()
    torch.cuda._sleep(2_000_000_000)            # about a second in which the queue fills up
    longest = 0.0
    for _ in range(20000):
        began = time.perf_counter()
        call()
        longest = max(longest, time.perf_counter() - began)
        if longest > 0.2:
            break
    done.set()
    other.join()
    torch.cuda.synchronize()
    assert longest > 0.2                        # a call did wait, ...
    assert max(gaps) < longest / 2, (max(gaps), longest)   # ... and the other thread did not
