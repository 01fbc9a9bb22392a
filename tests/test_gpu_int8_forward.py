"""Products of 8-bit codes with a scale for each token and channel: bit for bit the exact integer sum, rounded to binary32,
times the two scales there, rounded to 16 bits."""
import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, padded, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def codes(shape, seed, low=-128, high=128):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(low, high, shape, generator=g, device="cuda", dtype=torch.int8)


def scales(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    return torch.rand(n, generator=g, device="cuda") * 0.01 + 0.001


def product(x, w, sx, sw):
    return (x.double() @ w.double().T).float() * sx[:, None] * sw[None, :]     # sums below 2^53: exact


def check(wq, ctx, T, R, C, dtype, seed=0):  # noqa: F811
    x, w, sx, sw = codes((T, C), seed), codes((R, C), seed + 1), scales(T, seed), scales(R, seed + 2)
    want = product(x, w, sx, sw).to(dtype)
    out, whole = padded(torch.zeros((T, R), dtype=dtype, device="cuda"), 8, 3.0)
    # what lies behind a row does not enter a sum
    got = wq.windq_int8_forward(ctx, padded(x, 16, 113)[0], sx, padded(w, 16, -99)[0], sw, dtype=dtype, out=out)
    assert torch.equal(got, want)
    assert bool((whole[:, R:] == 3).all())


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 64, 65, 129, 200, 256, 257, 300, 320, 321, 400, 511, 700, 1025])
@pytest.mark.parametrize("R,C,dtype", [(128, 256, HALF), (1, 1, BF), (77, 2065, BF), (530, 131, HALF), (1000, 4096, BF)])
def test_sizes(wq, ctx, T, R, C, dtype):  # noqa: F811
    check(wq, ctx, T, R, C, dtype, seed=T + R)


@pytest.mark.parametrize("T,R,C", [(1, 14336, 4096), (7, 4096, 14336), (60, 512, 14336), (3, 100, 30000), (48, 11008, 4096), (203, 8192, 1024), (256, 2048, 8192),
                                   (777, 5120, 2824), (2000, 2056, 1000), (5000, 4093, 300), (600, 512, 16384)])
def test_larger_sizes(wq, ctx, T, R, C):  # noqa: F811
    check(wq, ctx, T, R, C, BF if T % 2 else HALF, seed=3)


@pytest.mark.parametrize("T", [2, 300, 400])
def test_the_longest_sum_of_the_lowest_codes(wq, ctx, T):  # noqa: F811
    C = 131071
    x = torch.full((T, C + 1), -128, dtype=torch.int8, device="cuda")[:, :C]
    w = torch.full((5, C + 1), -128, dtype=torch.int8, device="cuda")[:, :C]
    one = torch.full((T,), 2.0 ** -20, device="cuda")
    got = wq.windq_int8_forward(ctx, x, one, x[:5] if T >= 5 else w, torch.ones(5, device="cuda"), dtype=BF)
    assert bool((got.float() == torch.tensor(16384.0 * C * 2.0 ** -20).to(BF).float().item()).all())
    wide = torch.zeros((T, C + 17), dtype=torch.int8, device="cuda")
    with pytest.raises(wq.WindqError) as e:
        wq.windq_int8_forward(ctx, wide[:, :C + 1], one, wide[:, :C + 1], one, dtype=BF)
    assert e.value.status == 2


@pytest.mark.parametrize("T", [5, 500])
def test_a_scale_that_is_not_finite_spoils_its_row_or_column_alone(wq, ctx, T):  # noqa: F811
    x, w, sx, sw = codes((T, 96), 1), codes((70, 96), 2), scales(T, 1), scales(70, 2)
    sx[3], sw[66] = float("nan"), float("inf")
    got = wq.windq_int8_forward(ctx, x, sx, w, sw).isfinite()
    want = torch.ones((T, 70), dtype=torch.bool, device="cuda")
    want[3], want[:, 66] = False, product(x, w, sx, sw)[:, 66].isfinite()
    assert torch.equal(got, want)


def test_scales_start_anywhere(wq, ctx):  # noqa: F811
    for T in (9, 600):
        x, w, sx, sw = codes((T, 64), 1), codes((90, 64), 2), scales(T + 3, 1), scales(93, 2)
        for k in (1, 2, 3):
            a, b = sx[k:k + T], sw[k:k + 90]
            assert torch.equal(wq.windq_int8_forward(ctx, x, a, w, b), product(x, w, a, b).half())


def test_no_tokens(wq, ctx):  # noqa: F811
    assert wq.windq_int8_forward(ctx, codes((0, 64), 1), scales(0, 1), codes((8, 64), 2), scales(8, 1)).shape == (0, 8)


def test_equal_calls_give_equal_bits_on_other_streams_and_in_graphs(wq, ctx):  # noqa: F811
    x, w, sx, sw = codes((40, 8192), 1), codes((512, 8192), 2), scales(40, 1), scales(512, 2)
    want = wq.windq_int8_forward(ctx, x, sx, w, sw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(want)
    wq.windq_int8_forward(ctx, x, sx, w, sw, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    X = torch.randn((40, 8192), device="cuda").half()
    with torch.cuda.graph(graph):
        q = wq.windq_quantize_rows(ctx, X)
        y = wq.windq_int8_forward(ctx, q["codes"], q["scale"], w, sw)
    for seed in (5, 6):
        X.copy_(torch.randn((40, 8192), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        e = wq.windq_quantize_rows(ctx, X)
        assert torch.equal(y, wq.windq_int8_forward(ctx, e["codes"], e["scale"], w, sw))


def test_refusals(wq, ctx):  # noqa: F811
    x, w, sx, sw = codes((4, 64), 1), codes((8, 64), 2), scales(4, 1), scales(8, 2)
    call = lambda **k: wq.windq_int8_forward(ctx, *(dict(x=x, sx=sx, w=w, sw=sw) | k).values())  # noqa: E731
    for wrong in (dict(x=x.half()), dict(w=w.to(torch.uint8)), dict(sx=sx.half()), dict(x=x.cpu())):
        with pytest.raises(TypeError):
            call(**wrong)
    for wrong in (dict(x=x[:, :48]), dict(sx=sx[:3]), dict(sw=sw[::2]), dict(w=w.T), dict(x=x[0])):
        with pytest.raises(ValueError):
            call(**wrong)
    with pytest.raises(TypeError):
        wq.windq_int8_forward(ctx, x, sx, w, sw, dtype=torch.float32)
    with pytest.raises(ValueError):
        wq.windq_int8_forward(ctx, x, sx, w, sw, out=torch.empty((4, 9), dtype=HALF, device="cuda"))
    odd = torch.zeros((4, 72), dtype=torch.int8, device="cuda")
    for wrong in (dict(x=odd[:, :64]), dict(x=torch.zeros((4, 96), dtype=torch.int8, device="cuda")[:, 8:72])):
        with pytest.raises(wq.WindqError) as e:
            call(**wrong)
        assert e.value.status == 3
    out = torch.full((4, 12), 7.0, dtype=HALF, device="cuda")
    with pytest.raises(wq.WindqError):
        wq.windq_int8_forward(ctx, x, sx, w, sw, out=out[:, :8])
    torch.cuda.synchronize()
    assert bool((out == 7).all())
