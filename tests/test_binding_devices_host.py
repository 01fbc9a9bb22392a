"""Tensors on another device than the context's are refused before anything is launched.  Needs no GPU: the tensors are host
ones that name a device."""
import types

import pytest
import torch

HALF = torch.float16


class On(torch.Tensor):
    """A host tensor that says it lies on a CUDA device."""
    where = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.where

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        return args[0].where if func is torch.Tensor.get_device else super().__torch_function__(func, types, args, kwargs)


def on(t, device):
    t = t.as_subclass(On)
    t.where = device
    return t


class Library:
    """Counts the calls that reach the library."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


@pytest.fixture
def wq(monkeypatch):
    import paper_2605_26660_b200 as wq
    library = Library()
    monkeypatch.setattr(wq, "_lib", library)
    monkeypatch.setattr(wq, "_raw_stream", lambda ctx, stream: 0)
    wq_library = types.SimpleNamespace(wq=wq, library=library)
    return wq_library


CTX = types.SimpleNamespace(device=0, _h=None, _check=lambda st: None)


def lora():
    return dict(X=on(torch.zeros(4, 16, dtype=HALF), 0), W=on(torch.zeros(8, 16, dtype=HALF), 0), A=on(torch.zeros(2, 8, 16, dtype=HALF), 0),
                B=on(torch.zeros(2, 8, 8, dtype=HALF), 0), scaling=on(torch.zeros(2), 0), adapter_of=on(torch.zeros(4, dtype=torch.int32), 0))


def test_adapter_calls(wq):
    wq, library = wq.wq, wq.library
    out, dY = on(torch.zeros(4, 8, dtype=HALF), 0), on(torch.zeros(4, 8, dtype=HALF), 0)
    grads = dict(dx=on(torch.zeros(4, 16, dtype=HALF), 0), dA=on(torch.zeros(2, 8, 16), 0), dB=on(torch.zeros(2, 8, 8), 0))
    wq.windq_lora_forward(CTX, **lora(), out=out)
    wq.windq_lora_backward(CTX, **lora(), dY=dY, out=grads)
    assert library.calls == 2
    for key in lora():
        q = lora()
        q[key].where = 1
        with pytest.raises(ValueError, match="device"):
            wq.windq_lora_forward(CTX, **q, out=out)
        with pytest.raises(ValueError, match="device"):
            wq.windq_lora_backward(CTX, **q, dY=dY, out=grads)
    for t in (out, dY, *grads.values()):
        t.where = 1
        with pytest.raises(ValueError, match="device"):
            wq.windq_lora_forward(CTX, **lora(), out=out)
            wq.windq_lora_backward(CTX, **lora(), dY=dY, out=grads)
        t.where = 0
    assert library.calls == 6     # the forward calls before the four backward ones that were refused
    with pytest.raises(TypeError):
        wq.windq_lora_forward(CTX, **dict(lora(), A=torch.zeros(2, 8, 16, dtype=HALF)))


def states(n=300):
    new = lambda dt, k=n: on(torch.zeros(k, dtype=dt), 0)  # noqa: E731
    return dict(params=[new(torch.float32), new(torch.float32)], grads=[new(HALF), new(HALF)], m=[new(torch.int8), new(torch.int8)],
                v=[new(torch.uint8), new(torch.uint8)], m_scale=[new(torch.float32, 2), new(torch.float32, 2)],
                r_scale=[new(torch.float32, 2), new(torch.float32, 2)], copies=[new(HALF), new(HALF)])


def test_optimiser_calls(wq):
    wq, library = wq.wq, wq.library
    tensors = wq.AdamwTensors(**states())
    one, outs = on(torch.zeros(1), 0), ([on(torch.zeros(300), 0) for _ in range(2)], [on(torch.zeros(300), 0) for _ in range(2)])
    wq.windq_adamw_step(CTX, tensors, step=1, lr=1e-3, grad_scale=one)
    wq.windq_adamw_states(CTX, tensors, *outs)
    assert library.calls == 2
    for key in states():
        given = states()
        given[key][1].where = 1
        with pytest.raises(ValueError, match="device"):
            wq.AdamwTensors(**given)
    with pytest.raises(ValueError, match="device"):
        tensors.set_grads([on(torch.zeros(300, dtype=HALF), 1)] * 2)
    one.where = 1
    with pytest.raises(ValueError, match="device"):
        wq.windq_adamw_step(CTX, tensors, step=1, lr=1e-3, grad_scale=one)
    outs[1][1].where = 1
    with pytest.raises(ValueError, match="device"):
        wq.windq_adamw_states(CTX, tensors, *outs)
    other = types.SimpleNamespace(**dict(vars(CTX), device=1))
    with pytest.raises(ValueError, match="device"):
        wq.windq_adamw_step(other, tensors, step=1, lr=1e-3)
    with pytest.raises(ValueError, match="device"):
        wq.windq_adamw_states(other, tensors)
    assert library.calls == 2
