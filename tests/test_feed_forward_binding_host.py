"""What the compiled marshalling of the feed-forward calls refuses, before the library is reached.  Needs no GPU: every tensor
here is a host one, and a context without a library handle stands for the device."""
import types

import pytest
import torch

import paper_2605_26660_b200 as wq

CTX = types.SimpleNamespace(device=0, _h=types.SimpleNamespace(value=None), _check=None)
STREAM = types.SimpleNamespace(cuda_stream=0)
X, W = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(8, 64, dtype=torch.float16)
Q, P = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(8, 64, dtype=torch.int8)
S, R = torch.zeros(4), torch.zeros(8)
CALLS = {
    "quantize": lambda **k: wq.windq_quantize_rows(CTX, k.get("X", X), stream=STREAM),
    "int8": lambda **k: wq.windq_int8_forward(CTX, k.get("X", Q), S, P, R, dtype=k.get("dtype", torch.float16), stream=STREAM),
    "gated": lambda **k: wq.windq_gated_forward(CTX, k.get("X", X), W, W, activation=k.get("activation", "silu"), stream=STREAM),
    "gated_int8": lambda **k: wq.windq_gated_int8_forward(CTX, k.get("X", Q), S, P, R, P, R, activation=k.get("activation", "silu"), stream=STREAM),
    "backward": lambda **k: wq.windq_gated_backward(CTX, k.get("X", X), W, W, X, activation=k.get("activation", "gelu"), stream=STREAM),
}


@pytest.mark.parametrize("call", CALLS)
def test_host_tensors_and_other_types_are_refused(call):
    with pytest.raises(TypeError, match="must be a CUDA tensor"):
        CALLS[call]()
    with pytest.raises(TypeError, match="must be"):
        CALLS[call](X=X.double())
    with pytest.raises(TypeError, match="must be a tensor"):
        CALLS[call](X=[1.0])


@pytest.mark.parametrize("call", ["gated", "gated_int8", "backward"])
def test_unknown_activations_are_refused(call):
    with pytest.raises(ValueError, match="activation"):
        CALLS[call](activation="tanh")


def test_functions_count_their_arguments():
    with pytest.raises(TypeError, match="arguments"):
        wq._binding.quantize_rows(None, 0, STREAM, X)


def test_scratch_for_more_tokens_is_never_less():
    """So that what is reserved for the longest batch serves every shorter one, captured or not."""
    for bytes_of in (lambda T: wq.windq_scratch_bytes_int8_forward(T, 512, 512), lambda T: wq.windq_scratch_bytes_gated_forward(T, 512, 512),
                     lambda T: wq.windq_scratch_bytes_gated_backward(T, 512, 512), lambda T: wq.windq_scratch_bytes_gated_backward(T, 512, 512, True)):
        sizes = [bytes_of(T) for T in range(0, 1100)]
        assert sizes == sorted(sizes)
    assert wq.windq_scratch_bytes_int8_forward(-1, 5, 5) == 0 and wq.windq_scratch_bytes_gated_forward(4, 0, 5) == 0


def test_a_missing_context_is_refused_by_the_library():
    lib = wq._lib
    for status in (lib.windq_quantize_rows(None, 0, None, 4, 64, 64, None, 64, None, None, 0, None),
                   lib.windq_int8_forward(None, None, 4, 64, 64, None, None, 8, 64, None, 0, None, 8, None),
                   lib.windq_gated_forward(None, 0, 0, None, 4, 64, 64, None, 64, None, 64, 8, None, 8, None, None, 0, None),
                   lib.windq_gated_int8_forward(None, 0, None, 4, 64, 64, None, None, 64, None, None, 64, None, 8, 0, None, 8, None),
                   lib.windq_gated_backward(None, 0, 0, None, 4, 64, 64, None, 64, None, 64, 8, None, None, 8, None, 8, None, 64, None, None,
                                            64, None)):
        assert status == 1 and b"ctx is NULL" in lib.windq_last_error(None)
