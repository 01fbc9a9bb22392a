"""What AdamwTensors holds on the host: the memory whose addresses it hands to the library.  Needs no GPU: the tensors lie
in host memory that numpy owns, so that a weak reference tells whether it is still held, and the check that they are on a
device is left out."""
import gc
import weakref

import numpy as np
import pytest
import torch


@pytest.fixture
def wq(monkeypatch):
    import paper_2605_26660_b200 as wq
    monkeypatch.setattr(wq, "_need", lambda t, dtype, name, dims=None: t)
    return wq


def lists(n, bits):
    """The lists of one tensor each, and a weak reference to the memory of each."""
    state = (np.int8, np.uint8) if bits == 8 else (np.float32, np.float32)
    types = dict(params=np.float32, grads=np.float32, m=state[0], v=state[1], copies=np.float16)
    if bits == 8:
        types.update(m_scale=np.float32, r_scale=np.float32)
    given, memory = {}, {}
    for k, dt in types.items():
        a = np.zeros(-(-n // 256) if k.endswith("scale") else n, dt)
        given[k], memory[k] = [torch.from_numpy(a)], weakref.ref(a)
    return given, memory


def freed(memory):
    gc.collect()
    return [k for k, r in memory.items() if r() is None]


@pytest.mark.parametrize("bits", [32, 8])
def test_cleared_lists_free_nothing(wq, bits):
    given, memory = lists(1000, bits)
    held = wq.AdamwTensors(**given)
    for ts in given.values():
        ts.clear()
    assert freed(memory) == []
    del held
    assert len(freed(memory)) == len(memory)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_given_other_memory_keeps_the_old(wq, bits):
    # module.half() and the like put other memory under the same tensor object
    given, memory = lists(1000, bits)
    held = wq.AdamwTensors(**given)
    for ts in given.values():
        ts[0].data = torch.zeros(4, dtype=ts[0].dtype)
    assert freed(memory) == []
    del held


def test_gradients_are_held_until_others_come(wq):
    given, memory = lists(1000, 32)
    held = wq.AdamwTensors(**given)
    a = np.ones(1000, np.float32)
    grads, other = [torch.from_numpy(a)], weakref.ref(a)
    del a
    held.set_grads(grads)
    for ts in (grads, given["grads"]):
        ts.clear()
    assert freed(memory) == ["grads"] and other() is not None
