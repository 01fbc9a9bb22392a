"""Rows as 8-bit codes with one scale each: codes, scales and values against their definition in 64 bits, bit for bit.

127 x / a in binary64 is rounded once, and for 16-bit x and a no such quotient but a tie itself comes closer than 2^-18 of its
size to a border between two codes, so rounding it again to a code is rounding the exact quotient."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HALF, BF = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wq():
    import paper_2605_26660_b200 as wq
    return wq


@pytest.fixture(scope="module")
def ctx(wq):
    c = wq.windq_create()
    yield c
    wq.windq_destroy(c)


def definition(X):
    x = X.double()
    a = x.abs().amax(dim=1)
    q = torch.where(a[:, None] > 0, torch.round(127 * x / torch.where(a > 0, a, 1.0)[:, None]), 0.0)
    scale = (a / 127).float()                          # a has 11 bits: the quotient is not near a border of binary32 twice
    return q.to(torch.int8), scale, (q.float() * scale[:, None]).to(X.dtype)


def padded(X, step, fill):
    T, C = X.shape
    whole = torch.full((T, C + -C % step + step), fill, dtype=X.dtype, device="cuda")
    whole[:, :C] = X
    return whole[:, :C], whole


def check(wq, ctx, X):
    T, C = X.shape
    view, _ = padded(X, 8, float("nan"))               # what lies behind a row is not read
    codes, codes_whole = padded(torch.zeros((T, C), dtype=torch.int8, device="cuda"), 16, 77)
    values, values_whole = padded(torch.zeros_like(X), 8, 5.0)
    got = wq.windq_quantize_rows(ctx, view, want_values=True, out=dict(codes=codes, values=values))
    q, scale, v = definition(X)
    assert torch.equal(got["codes"], q)
    assert torch.equal(got["scale"], scale)
    assert torch.equal(got["values"], v)
    assert bool((codes_whole[:, C:] == 77).all()) and bool((values_whole[:, C:] == 5).all())
    again = wq.windq_quantize_rows(ctx, view)
    assert torch.equal(again["codes"], q) and again["values"] is None
    assert again["codes"].stride(0) % 16 == 0


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("T,C", [(1, 1), (1, 7), (3, 8), (1, 2048), (1, 14336), (5, 130), (70, 2049), (300, 4096), (9, 8200), (2500, 1000),
                                 (33, 16390), (2, 40003), (9000, 24), (2400, 5000), (1200, 11008)])
def test_codes_scales_and_values(wq, ctx, T, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(T * 7 + C)
    X = torch.randn((T, C), generator=g, device="cuda") * torch.randn((T, 1), generator=g, device="cuda").exp()
    X[torch.rand((T, C), generator=g, device="cuda") < 0.1] = 0
    check(wq, ctx, X.to(dtype))


@pytest.mark.parametrize("dtype", [HALF, BF])
def test_every_value_below_a_maximum(wq, ctx, dtype):
    """All finite values of the type up to each of 64 maxima, the extremes among them: ties and all."""
    top = 0x7c00 if dtype is HALF else 0x7f80
    bits = torch.arange(top, dtype=torch.int32, device="cuda")
    one = bits.to(torch.int16).view(dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    maxima = torch.randint(1, top, (64,), generator=g, device="cuda")
    maxima[:8] = torch.tensor([1, 2, 3, 127, 128, 255, top - 1, top // 2], device="cuda")
    # ties need maxima of few bits: powers of two times 1, 127 / 64, 3, 5
    maxima[8:12] = torch.tensor([1.0, 127 / 64, 3.0, 5.0], device="cuda").to(dtype).view(torch.int16).int()
    X = torch.where(bits[None, :] <= maxima[:, None], one[None, :].expand(64, -1), torch.zeros((), dtype=dtype, device="cuda"))
    check(wq, ctx, torch.cat([X, -X], dim=1).contiguous())


def test_ties_go_to_even(wq, ctx):
    # a = 127: the codes are the values themselves, halves are ties
    X = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 63.5, 64.5, -126.5, 0.25, -0.75]], device="cuda")
    for dtype in (HALF, BF):
        got = wq.windq_quantize_rows(ctx, X.to(dtype)[:, :9].contiguous()[:, :8])["codes"]
        assert got[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 64]
        check(wq, ctx, X.to(dtype))


@pytest.mark.parametrize("dtype", [HALF, BF])
def test_rows_of_zeros_and_rows_that_are_not_finite(wq, ctx, dtype):
    X = torch.randn((6, 300), device="cuda").to(dtype)
    X[1], X[2, 299], X[3, 0], X[4, 17] = 0, float("inf"), float("-inf"), float("nan")
    got = wq.windq_quantize_rows(ctx, padded(X, 8, 0)[0], want_values=True)
    fine = [0, 1, 5]
    q, scale, v = definition(X[fine])
    assert torch.equal(got["codes"][fine], q) and torch.equal(got["scale"][fine], scale) and torch.equal(got["values"][fine], v)
    assert float(got["scale"][1]) == 0
    assert bool((got["codes"][2:5] == 0).all()) and bool(got["scale"][2:5].isnan().all()) and bool(got["values"][2:5].isnan().all())


def test_scales_start_anywhere_and_no_rows_are_no_work(wq, ctx):
    X = torch.randn((5, 64), device="cuda").half()
    q, scale, _ = definition(X)
    for first in (1, 2, 3):
        s = torch.full((first + 6,), 9.0, device="cuda")
        got = wq.windq_quantize_rows(ctx, X, out=dict(scale=s[first:first + 5]))
        assert torch.equal(got["codes"], q) and torch.equal(s[first:first + 5], scale) and float(s[first + 5]) == 9
    got = wq.windq_quantize_rows(ctx, X[:0], want_values=True)
    assert got["codes"].shape == (0, 64) and got["scale"].shape == (0,)


def test_a_long_tensor_passes_32_bits_of_offset(wq, ctx):
    T, C = 70000, 32768                                    # 2.3e9 values
    X = torch.zeros((T, C), dtype=HALF, device="cuda")
    X[-3:] = torch.randn((3, C), device="cuda").half()
    got = wq.windq_quantize_rows(ctx, X)
    q, scale, _ = definition(X[-3:])
    assert torch.equal(got["codes"][-3:], q) and torch.equal(got["scale"][-3:], scale)
    assert float(got["scale"][:-3].max()) == 0


def test_refusals(wq, ctx):
    X = torch.zeros((4, 64), dtype=HALF, device="cuda")
    with pytest.raises(TypeError):
        wq.windq_quantize_rows(ctx, X.float())
    with pytest.raises(TypeError):
        wq.windq_quantize_rows(ctx, X.cpu())
    with pytest.raises(ValueError):
        wq.windq_quantize_rows(ctx, X.T)
    with pytest.raises(ValueError):
        wq.windq_quantize_rows(ctx, X, out=dict(codes=torch.empty((4, 63), dtype=torch.int8, device="cuda")))
    with pytest.raises(ValueError):
        wq.windq_quantize_rows(ctx, X, out=dict(scale=torch.empty(3, device="cuda")))
    for bad, status in ((X[:, 1:33], 3), (X[:, :0], 2), (torch.zeros((4, 60), dtype=HALF, device="cuda"), 3)):
        with pytest.raises(wq.WindqError) as e:
            wq.windq_quantize_rows(ctx, bad)
        assert e.value.status == status
    with pytest.raises(wq.WindqError) as e:
        wq.windq_quantize_rows(ctx, X, out=dict(codes=torch.empty((4, 72), dtype=torch.int8, device="cuda")[:, :64]))
    assert e.value.status == 3
