"""The counters of a context tell of every call issued before they are asked, on whatever stream it runs."""
import ctypes

import pytest
import torch

import windq_synth as ws
from test_gpu_lora import HALF, backward, ctx, forward, inputs, wq  # noqa: F401

pytestmark = pytest.mark.gpu

CYCLES = 200_000_000   # a tenth of a second of work before the call


def test_fit_work_counts_a_call_that_has_not_started(wq):  # noqa: F811
    own, side = wq.windq_create(0), torch.cuda.Stream()
    W, s, grid = ws.weights(256, 512, 1, "student_t").cuda(), torch.ones(512, device="cuda"), torch.from_numpy(ws.clip_grid(20)).cuda()
    wq.windq_fit_eval(own, W, 128, s, grid)
    _, searched = wq.windq_fit_work(own, reset=True)
    assert searched > 0
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
        wq.windq_fit_eval(own, W, 128, s, grid)
    assert wq.windq_fit_work(own, reset=True)[1] == searched and side.query()
    assert wq.windq_fit_work(own)[1] == 0
    wq.windq_destroy(own)


def test_stalls_are_asked_after_the_calls_before(wq, ctx):  # noqa: F811
    q, _ = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=60)
    forward(wq, ctx, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
        forward(wq, ctx, q)
    assert wq.windq_stalls(ctx) == 0 and side.query()


class _Head(ctypes.Structure):
    """The first members of windq_ctx."""
    _fields_ = [("device", ctypes.c_int), ("sm_count", ctypes.c_int), ("gave_up", ctypes.POINTER(ctypes.c_uint))]


def test_after_a_wait_that_gave_up_the_calls_refuse(wq):  # noqa: F811
    # the failure is made on the host: the word a kernel would write is written here
    own = wq.windq_create(0)
    q, dY = inputs(24, 264, 520, 16, 4, HALF, "mixed", seed=61)
    y = forward(wq, own, q)
    head = _Head.from_address(own._h.value)
    assert head.device == 0 and head.sm_count == torch.cuda.get_device_properties(0).multi_processor_count and head.gave_up[0] == 0
    head.gave_up[0] = 1
    out = torch.full_like(y, 7)
    for call in (lambda: forward(wq, own, q, out=out), lambda: backward(wq, own, q, dY)):
        with pytest.raises(wq.WindqError, match="gave up") as e:
            call()
        assert e.value.status == 6
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    assert wq.windq_stalls(own) == 0 and head.gave_up[0] == 1      # asking alone does not forget it
    wq.windq_stalls(own, reset=True)
    assert torch.equal(forward(wq, own, q), y)
    wq.windq_destroy(own)
