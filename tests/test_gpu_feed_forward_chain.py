"""A whole training step and a served batch without a pause between the calls: every kernel starts while the one before ends, and
must not read what that still writes.  The same calls with a wait after each give the bits to compare with."""
import pytest
import torch

from test_gpu_quantize_rows import BF, HALF, ctx, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def make(T, C, F, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return dict(X=r(T, C).to(dtype), Wg=(0.1 * r(F, C)).to(dtype), Wu=(0.1 * r(F, C)).to(dtype), Wd=(0.05 * r(C, F)).to(dtype),
                A=(0.1 * r(2, 16, F)).to(dtype), B=(0.1 * r(2, C, 16)).to(dtype), scaling=torch.ones(2, device="cuda"),
                ids=torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda").repeat(T // 3 + 1)[:T].contiguous(), want=r(T, C))


def same(a, b):
    """Bit for bit: where gradients leave fp16's range, infinities and what comes of them are results like others."""
    return torch.equal(a.view(torch.int32 if a.dtype == torch.float32 else torch.int16), b.view(torch.int32 if b.dtype == torch.float32 else torch.int16))


def step(wq, c, s, wait, rounds, loss=1.0):  # noqa: F811
    """Training steps of the block with an adapted down projection, then a pass in 8 bits through what came out."""
    s = {k: v.clone() for k, v in s.items()}
    copies = [s["Wg"], s["Wu"], s["A"], s["B"]]
    master = [w.float() for w in copies]
    grads = [torch.zeros_like(w) for w in copies]
    slow = [torch.zeros(w.shape, device="cuda") for w in copies[2:]]
    tensors = wq.AdamwTensors(master[:2], grads[:2], [torch.zeros_like(w) for w in master[:2]], [torch.zeros_like(w) for w in master[:2]],
                              copies=copies[:2])
    adapters = wq.AdamwTensors(master[2:], slow, [torch.zeros_like(w) for w in slow], [torch.zeros_like(w) for w in slow], copies=copies[2:])
    pause = torch.cuda.synchronize if wait else lambda: None
    dY = torch.empty_like(s["X"])
    for k in range(1, rounds + 1):
        f = wq.windq_gated_forward(c, s["X"], s["Wg"], s["Wu"], want_saved=True)
        pause()
        wq.windq_lora_forward(c, f["h"], s["Wd"], s["A"], s["B"], s["scaling"], s["ids"], out=dY)
        dY.mul_(loss)
        pause()
        b = wq.windq_lora_backward(c, f["h"], s["Wd"], s["A"], s["B"], s["scaling"], s["ids"], dY, out=dict(dA=slow[0], dB=slow[1]))
        pause()
        d = wq.windq_gated_backward(c, s["X"], s["Wg"], s["Wu"], b["dx"], gate=f["gate"], up=f["up"], out=dict(dWg=grads[0], dWu=grads[1]))
        pause()
        wq.windq_adamw_step(c, tensors, step=k, lr=1e-3)
        pause()
        wq.windq_adamw_step(c, adapters, step=k, lr=1e-3)
        pause()
    q = [wq.windq_quantize_rows(c, w) for w in (s["Wg"], s["Wu"], s["Wd"])]
    pause()
    x = wq.windq_quantize_rows(c, s["X"])
    pause()
    h = wq.windq_gated_int8_forward(c, x["codes"], x["scale"], q[0]["codes"], q[0]["scale"], q[1]["codes"], q[1]["scale"])
    pause()
    z = wq.windq_quantize_rows(c, h)
    pause()
    y = wq.windq_int8_forward(c, z["codes"], z["scale"], q[2]["codes"], q[2]["scale"])
    pause()
    return [f["h"], dY, d["dx"], *grads, *slow, *copies, h, y]


@pytest.mark.parametrize("T,C,F,dtype", [(1, 512, 1408, HALF), (40, 1024, 2048, BF), (64, 264, 520, HALF), (200, 2048, 1024, HALF),
                                         (700, 512, 1000, BF), (3000, 1024, 768, HALF)])
@pytest.mark.parametrize("loss", [1.0, 2.0 ** -8])
def test_calls_back_to_back(wq, ctx, T, C, F, dtype, loss):  # noqa: F811
    s = make(T, C, F, dtype, T)
    want = step(wq, ctx, s, True, 3, loss)
    assert loss == 1.0 or all(bool(t.isfinite().all()) for t in want)
    for _ in range(3):
        for k, (a, b) in enumerate(zip(step(wq, ctx, s, False, 3, loss), want)):
            assert same(a, b), k


def test_two_contexts_on_two_streams(wq):  # noqa: F811
    """Kernels of a few tokens, of pairs of whole SMs and of adapters side by side: nothing waits for what the other holds."""
    cases = [make(40, 1024, 2048, BF, 1), make(500, 1024, 1536, HALF, 2)]
    contexts = [wq.windq_create(), wq.windq_create()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = [step(wq, c, s, True, 2) for c, s in zip(contexts, cases)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k].append(step(wq, contexts[k], cases[k], False, 2))
    torch.cuda.synchronize()
    for k in (0, 1):
        for run in got[k]:
            assert all(same(a, b) for a, b in zip(run, want[k]))
        assert wq.windq_stalls(contexts[k]) == 0
        wq.windq_destroy(contexts[k])


@pytest.mark.parametrize("T,R,C", [(1, 4096, 2048), (20, 2048, 4096), (90, 3000, 1024), (300, 2048, 2048), (1000, 1024, 1024)])
def test_a_weight_that_the_kernel_before_still_writes(wq, ctx, T, R, C):  # noqa: F811
    """The product brings its first weights into L2 while the quantiser that writes them runs: it must multiply with what that leaves."""
    g = torch.Generator(device="cuda").manual_seed(T)
    weights = [torch.randn((R, C), generator=g, device="cuda").half() for _ in range(3)]
    x = wq.windq_quantize_rows(ctx, torch.randn((T, C), generator=g, device="cuda").half())
    want = []
    for w in weights:
        q = wq.windq_quantize_rows(ctx, w)
        torch.cuda.synchronize()
        want.append(wq.windq_int8_forward(ctx, x["codes"], x["scale"], q["codes"], q["scale"]))
        torch.cuda.synchronize()
    out = wq.windq_quantize_rows(ctx, weights[0])
    got = []
    for k in range(60):
        wq.windq_quantize_rows(ctx, weights[k % 3], out=out)
        got.append(wq.windq_int8_forward(ctx, x["codes"], x["scale"], out["codes"], out["scale"]))
    for k, y in enumerate(got):
        assert torch.equal(y, want[k % 3]), k
