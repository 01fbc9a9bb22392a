"""What the adapter calls take and refuse beyond test_gpu_lora.py."""
import ctypes

import pytest
import torch

from test_gpu_lora import BF, HALF, backward, ctx, exact, forward, inputs, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 40, 300, 700])
def test_adapter_of_and_scaling_start_anywhere(wq, ctx, T):  # noqa: F811
    q, dY = inputs(T, 136, 264, 16, 5, HALF, "mixed", seed=70)
    want = exact(q, dY)
    for first in (1, 2, 3):
        ids = torch.full((first + T,), -1, dtype=torch.int32, device="cuda")
        scaling = torch.full((first + 5,), 99.0, device="cuda")
        ids[first:], scaling[first:] = q["ids"], q["scaling"]
        p = dict(q, ids=ids[first:], scaling=scaling[first:])
        assert torch.equal(forward(wq, ctx, p), want["y"].to(HALF))
        back = backward(wq, ctx, p, dY)
        assert torch.equal(back["dx"], want["dx"].to(HALF))
        assert torch.equal(back["dA"], want["dA"].float()) and torch.equal(back["dB"], want["dB"].float())


def test_addresses_between_words_are_refused(wq, ctx):  # noqa: F811
    q, _ = inputs(8, 64, 64, 16, 3, HALF, "mixed", seed=71)
    y = torch.full((8, 64), 7.0, dtype=HALF, device="cuda")
    at = lambda t, k=0: ctypes.c_void_p(t.data_ptr() + k)  # noqa: E731
    for bad in ((2, 0), (0, 2), (1, 0)):
        status = wq._lib.windq_lora_forward(ctx._h, 0, at(q["X"]), 8, 64, 64, at(q["W"]), 64, 64, at(q["A"]), at(q["B"]), 3, 16,
                                            at(q["scaling"], bad[0]), at(q["ids"], bad[1]), at(y), 64, None)
        assert status == 3
    torch.cuda.synchronize()
    assert bool((y == 7).all())
