"""Every quotient 127 x / a of 16-bit x and a that decides a code, up to powers of two that cancel: the codes are those of the exact
quotient, rounded in integers.  The closest to a border between two codes, but for ties, is 127 * 2025 / 2033 = 126.50025, 2^-18.97 of
itself away from 126.5."""
import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bits", [(HALF, 11), (BF, 8)])
@pytest.mark.parametrize("power", [0, -3, 4])
def test_every_quotient(wq, ctx, dtype, bits, power):  # noqa: F811
    low = 1 << (bits - 1)
    a, m = torch.arange(low, 2 * low, device="cuda"), torch.arange(low, 2 * low, device="cuda")
    for shift in range(9):                     # x = m 2^-shift: below 2^-8 of a all codes are 0, or half of a step
        live = m[None, :] <= a[:, None] << shift
        x = torch.where(live, m[None, :], torch.zeros_like(m[None, :]))
        X = torch.cat([a[:, None].double(), x.double() * 2.0 ** -shift, -x.double() * 2.0 ** -shift], dim=1) * 2.0 ** power
        rows = torch.zeros((low, X.shape[1] + -X.shape[1] % 8), dtype=dtype, device="cuda")[:, :X.shape[1]]
        rows.copy_(X)
        assert bool((rows.double() == X).all())
        got = wq.windq_quantize_rows(ctx, rows)["codes"].long()
        n, d = 127 * x, a[:, None] << shift
        q = (2 * n + d) // (2 * d)             # half up, ...
        q = q - (((2 * n + d) % (2 * d) == 0) & (q % 2 == 1)).long()   # ... but for ties, which go to even
        assert bool((got[:, 0] == 127).all())
        assert torch.equal(got[:, 1:1 + low], q) and torch.equal(got[:, 1 + low:], -q)


def test_the_closest_of_all(wq, ctx):  # noqa: F811
    X = torch.tensor([[2033.0, 2025.0, -2025.0, 0, 0, 0, 0, 0]], device="cuda").half()
    assert wq.windq_quantize_rows(ctx, X)["codes"][0, :3].tolist() == [127, 127, -127]
