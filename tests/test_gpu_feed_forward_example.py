"""The example that quantises a gated block, trains it on and serves it in 8 bits: the operators working together."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def run():
    spec = importlib.util.spec_from_file_location("feed_forward", os.path.join(ROOT, "examples", "feed_forward.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example.main(verbose=False)


def test_its_first_gradients(run):
    losses, first, _ = run
    assert all(loss == loss and loss < float("inf") for loss in losses)
    x, dh = first["X"].double(), first["dH"].double()
    wg, wu = (first[k].double().requires_grad_(True) for k in ("Wg", "Wu"))
    (torch.nn.functional.silu(x @ wg.T) * (x @ wu.T) * dh).sum().backward()
    for name, w in (("dWg", wg), ("dWu", wu)):
        # the products kept in 16 bits, the terms' rounding and the result's: each half a step at most, independent of one another
        off = (first[name].double() - w.grad).norm() / w.grad.norm()
        assert float(off) < 3 * 2.0 ** -11, name


def dequantised(t):
    a = t.double().abs().amax(dim=1, keepdim=True)
    return torch.round(127 * t.double() / a) * a / 127


def test_what_it_serves(run):
    _, _, served = run
    x, (wg, wu, wd) = dequantised(served["X"]), (dequantised(w) for w in served["weights"])
    h = torch.nn.functional.silu(x @ wg.T) * (x @ wu.T)
    assert float((served["H"].double() - h).norm() / h.norm()) < 2.0 ** -11
    y = dequantised(served["H"]) @ wd.T
    assert float((served["Y"].double() - y).norm() / y.norm()) < 2.0 ** -11
