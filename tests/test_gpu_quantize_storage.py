"""Codes and scales are tensors of their own: keeping or saving one of them keeps nothing of the other."""
import io

import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,C,dtype", [(1, 2048, HALF), (4, 104, BF), (300, 1000, HALF), (1000, 4096, BF), (0, 64, HALF)])
def test_no_storage_is_shared(wq, ctx, T, C, dtype):  # noqa: F811
    got = wq.windq_quantize_rows(ctx, torch.randn((T, C), device="cuda").to(dtype), want_values=True)
    storages = {k: t.untyped_storage() for k, t in got.items()}
    assert storages["scale"].nbytes() == 4 * T
    if T:
        assert len({s.data_ptr() for s in storages.values()}) == 3
    saved = io.BytesIO()
    torch.save(got["scale"], saved)
    assert saved.tell() < 4 * T + 4096
    saved.seek(0)
    assert torch.equal(torch.load(saved), got["scale"])


def test_scales_outlive_their_codes(wq, ctx):  # noqa: F811
    W = torch.randn((4096, 4096), device="cuda").half()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    scale = wq.windq_quantize_rows(ctx, W)["scale"]
    assert torch.cuda.memory_allocated() - before <= 32768
    assert torch.equal(scale, (W.float().abs().amax(dim=1).double() / 127).float())
