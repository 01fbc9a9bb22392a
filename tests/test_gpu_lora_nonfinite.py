"""An adapter that diverged shows: where the formula gives no finite value the calls give none, on either type, and what
does not depend on the adapter keeps its exact value."""
import pytest
import torch

from test_gpu_lora import BF, HALF, backward, ctx, exact, forward, inputs, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def same(got, want, what):
    want = want.to(got.dtype)
    fine = want.isfinite()
    assert torch.equal(got.isfinite(), fine), what
    assert torch.equal(got[fine], want[fine]), what


def spoil(q, key, value):
    t = q[key]
    if key == "scaling":
        t[0] = value
    else:
        t[0, 5, 7] = value
    return q


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("key", ["A", "B", "scaling"])
@pytest.mark.parametrize("dt", [HALF, BF])
def test_an_adapter_that_is_not_finite_shows(wq, ctx, dt, key, value):  # noqa: F811
    # its tokens in a tile of their own, of which the header tells that an adapter may spoil it
    q, dY = inputs(600, 136, 264, 16, 3, dt, "mixed", seed=40)
    q["ids"] = torch.where(q["ids"] == 0, 1, q["ids"])
    q["ids"][:256] = 0
    spoil(q, key, value)
    want = exact(q, dY)
    same(forward(wq, ctx, q), want["y"], "y")
    back = backward(wq, ctx, q, dY)
    for k in ("dx", "dA", "dB"):
        same(back[k], want[k], k)
    assert not want["y"][:256].isfinite().all() and want["y"][256:].isfinite().all()


@pytest.mark.parametrize("T", [5, 150, 700])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dt", [HALF, BF])
def test_its_low_rank_values_stay_with_its_tokens(wq, ctx, dt, value, T):  # noqa: F811
    # the factor that makes u (or v) is not finite, the one u is taken times is: neighbours in the tile do not see it
    for key, results in (("A", ("y", "dB")), ("B", ("dx", "dA")), ("scaling", ("y", "dx", "dA", "dB"))):
        q, dY = inputs(T, 136, 264, 16, 3, dt, "mixed", seed=41)
        q["ids"][0] = 0
        want = exact(spoil(q, key, value), dY)
        got = dict(backward(wq, ctx, q, dY), y=forward(wq, ctx, q))
        for k in results:
            same(got[k], want[k], (key, k))
            assert not want[k].isfinite().all()
