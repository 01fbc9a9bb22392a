"""Cases and plain forms of the operators that tune and serve low-rank adapters over a quantised model.

Three operators, each through the package's public calls where ``own`` is set and in elementary torch operations in
32 bits where it is not:

  lora_forward   Y = X W^T + scaling[a] (X A_a^T) B_a^T, where a = adapter_of[t] is the adapter of token t (-1: none)
                 and W is the weight all requests share (as windq_apply_plan leaves it, fake-quantised)
  lora_backward  dX, dA, dB of the same for frozen W
  adamw          one AdamW step over all tensors of a set of adapters, states in 32 bits or in 8

The 8-bit states: every block of 256 elements of a tensor has one fp32 scale for m (its largest |m|) and one for
r = sqrt(v) (its largest r).  m stands for sign(q) (q / 127)^2 scale with q in [-127, 127], r for (q / 255)^2 scale
with q in [0, 255]; an r above zero never gets the code 0.
"""
import math
import random

import torch

own = False

BLOCK = 256                                   # elements of a tensor that share a state scale
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 2e-4, 0.01
TINY = 2.0 ** -100                            # a block whose largest value is below this is stored as zeros


def _lora(op, name, T, R, C, rank, adapters, requests, dtype):
    return {"name": name, "op": op, "T": T, "R": R, "C": C, "rank": rank, "adapters": adapters, "requests": requests,
            "dtype": dtype}


def _adamw(name, hidden, inter, kv, rank, blocks, odd, state, grad, copy):
    return {"name": name, "op": "adamw", "hidden": hidden, "inter": inter, "kv": kv, "rank": rank, "blocks": blocks,
            "odd": odd, "state": state, "grad": grad, "copy": copy}


def listed():
    return [
        # one user, one token, the query projection of a 1B-shaped model: launch latency
        _lora("lora_forward", "decode_one_token", 1, 2048, 2048, 16, 4, 1, "f16"),
        # a batch of requests, each with one of 32 adapters, the gate projection of a 7B-shaped model: memory
        _lora("lora_forward", "decode_48_requests", 48, 11008, 4096, 16, 32, 48, "bf16"),
        # a big batch of single tokens (or drafts to be verified), a 70B-shaped query projection
        _lora("lora_forward", "decode_203_requests", 203, 8192, 8192, 32, 48, 203, "f16"),
        # a few prompts of unequal length packed without padding, the down projection of a 13B-shaped model
        _lora("lora_forward", "prompts_ragged", 777, 5120, 13824, 8, 6, 9, "f16"),
        # long prompts, the gate projection of an 8B-shaped model: tensor cores
        _lora("lora_forward", "prompts_long", 8192, 14336, 4096, 64, 8, 5, "bf16"),
        # one short training sequence, the key projection of a 1B-shaped model: latency
        _lora("lora_backward", "backward_short", 96, 512, 2048, 8, 1, 1, "f16"),
        # several adapters trained at once on sequences of unequal length, the down projection of a 7B-shaped model
        _lora("lora_backward", "backward_ragged", 1531, 4096, 11008, 32, 3, 7, "bf16"),
        # a training batch of long sequences, the query projection of a 7B-shaped model
        _lora("lora_backward", "backward_long", 8192, 4096, 4096, 16, 2, 8, "f16"),
        # the adapters of one 1B-shaped block: 14 tensors, latency
        _adamw("adamw_block", 2048, 8192, 512, 8, 1, 0, "f32", "f32", "f16"),
        # the adapters of a whole 7B-shaped model (448 tensors, 160 M elements)
        _adamw("adamw_model", 4096, 11008, 4096, 64, 32, 0, "f32", "f32", "bf16"),
        # eight blocks with 8-bit states, 16-bit gradients, and a learned vector of odd length in each block
        _adamw("adamw_8bit_blocks", 2048, 8192, 512, 16, 8, 2049, "q8", "bf16", "none"),
        # the whole 7B-shaped model with 8-bit states
        _adamw("adamw_8bit_model", 4096, 11008, 4096, 64, 32, 0, "q8", "f32", "bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    x = min(max(x, lo), hi)
    return x + step if x == 3072 else x       # that size belongs to no model here


def draw(rng):
    op = rng.choice(["lora_forward", "lora_forward", "lora_backward", "adamw"])
    if op == "adamw":
        state = rng.choice(["f32", "q8"])
        return {"op": op, "hidden": _log_int(rng, 512, 8192, 8), "inter": _log_int(rng, 1024, 16384, 8),
                "kv": _log_int(rng, 128, 4096, 8), "rank": 8 * rng.randint(1, 4), "blocks": _log_int(rng, 1, 32),
                "odd": rng.choice([0, rng.randint(1, 5000)]), "state": state, "grad": rng.choice(["f32", "f16", "bf16"]),
                "copy": rng.choice(["none", "f16", "bf16"])}
    T = _log_int(rng, 1, 8192)
    R, C = _log_int(rng, 256, 14336, 8), _log_int(rng, 256, 14336, 8)
    while R * C > 14336 * 4096:
        R, C = max(256, R // 16 * 8), max(256, C // 16 * 8)
    if R == 3072 or C == 3072:
        R, C = R + 8, C + 8
    rank = rng.choice([8, 16, 16, 24, 32, 64, 128])
    adapters = _log_int(rng, 1, 32)
    requests = T if op == "lora_forward" and T <= 256 and rng.random() < 0.7 else rng.randint(1, min(T, 12))
    return {"op": op, "T": T, "R": R, "C": C, "rank": rank, "adapters": adapters, "requests": requests,
            "dtype": rng.choice(["f16", "bf16"])}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _lora_inputs(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    T, R, C, r, n, dt = case["T"], case["R"], case["C"], case["rank"], case["adapters"], DTYPES[case["dtype"]]
    x = _randn((T, C), g) * (0.5 * _randn((C,), g)).exp_()        # channels of unequal scale ...
    x[:, torch.randint(0, C, (4,), generator=g, device="cuda")] *= 20.0          # ... and a few hot ones
    step = 0.005 + 0.005 * torch.rand((R, 1), generator=g, device="cuda")        # a quantised weight: few levels a row
    w = _randn((R, C), g).mul_(0.02).div_(step).round_().mul_(step)
    s = {"X": x.to(dt), "W": w.to(dt), "A": (_randn((n, r, C), g) / math.sqrt(C)).to(dt),
         "B": (0.02 * _randn((n, R, r), g)).to(dt), "rank": r}
    s["scaling"] = torch.tensor([rng.choice([0.5, 1.0, 2.0]) for _ in range(n)], dtype=torch.float32).cuda()
    # requests one after another, an adapter (or, one time in eight, none) to each
    q = case["requests"]
    cuts = list(range(T + 1)) if q == T else [0] + sorted(rng.randint(0, T) for _ in range(q - 1)) + [T]
    ids = [-1 if q > 1 and rng.random() < 0.125 else rng.randrange(n) for _ in range(q)]
    lengths = torch.tensor([b - a for a, b in zip(cuts, cuts[1:])])
    s["adapter_of"] = torch.repeat_interleave(torch.tensor(ids, dtype=torch.int32), lengths).cuda()
    if case["op"] == "lora_backward":
        s["dY"] = (0.01 * _randn((T, R), g)).to(dt)
    return s


def _shapes(case):
    h, i, kv, r = case["hidden"], case["inter"], case["kv"], case["rank"]
    sizes = []
    for _ in range(case["blocks"]):
        for R, C in ((h, h), (kv, h), (kv, h), (h, h), (i, h), (i, h), (h, i)):
            sizes += [r * C, r * R]
        if case["odd"]:
            sizes.append(case["odd"])
    return sizes


def _layout(case):
    """(elements, first element) of every tensor in one arena, each on a whole block, and the arena's size."""
    sizes, first, at = _shapes(case), [], 0
    for n in sizes:
        first.append(at)
        at += -(-n // BLOCK) * BLOCK
    return sizes, first, at


def _encode(x, levels, signed):
    """Codes and scales of 8-bit states, for whole blocks of x."""
    a = x.abs().view(-1, BLOCK)
    top = a.amax(dim=1)
    top = torch.where(top >= TINY, top, torch.zeros_like(top))
    inv = torch.where(top > 0, torch.reciprocal(top), torch.zeros_like(top))
    q = ((a * inv[:, None]).sqrt() * float(levels)).round()
    q = q.clamp(max=float(levels))
    if signed:
        return (q * torch.sign(x.view(-1, BLOCK))).to(torch.int8).view(-1), top
    q = torch.where((a > 0) & (top > 0)[:, None], q.clamp(min=1.0), q)
    return q.to(torch.uint8).view(-1), top


def _decode(q, scale, levels):
    u = q.to(torch.float32) * torch.tensor(1.0 / levels, dtype=torch.float32).item()
    return ((u * u.abs()).view(-1, BLOCK) * scale[:, None]).view(-1)


def _adamw_inputs(case, seed):
    g = _gen(seed)
    sizes, first, total = _layout(case)
    live = torch.zeros(total + 1, dtype=torch.int8, device="cuda")     # 1 inside a tensor, 0 in the padding between
    edge = torch.tensor([first, [a + n for a, n in zip(first, sizes)]], device="cuda")
    live[edge[0]] += 1
    live.index_add_(0, edge[1], torch.full_like(edge[1], -1, dtype=torch.int8))
    live = live[:total].cumsum(0, dtype=torch.int8).to(torch.bool)
    width = (0.7 * _randn((total // BLOCK, 1), g)).exp_()              # gradients of unequal size across a model
    like = lambda k: (_randn((total // BLOCK, BLOCK), g) * width * k).view(-1) * live  # noqa: E731
    s = {"param": like(0.02), "grad": like(1e-3).to(DTYPES[case["grad"]]), "step": 10, "sizes": sizes, "first": first}
    m, r = like(3e-4), (like(1e-3).square_() + like(3e-4).square_()).sqrt_()
    if case["state"] == "q8":
        m[: BLOCK] = 0.0                                               # a block whose state is still empty
        r[: BLOCK] = 0.0
        s["m"], s["m_scale"] = _encode(m, 127, True)
        s["r"], s["r_scale"] = _encode(r, 255, False)
        s["m_value"], s["v_value"] = torch.empty_like(m), torch.empty_like(m)
    else:
        s["m"], s["v"] = m, r.square_()
    s["copy"] = None if case["copy"] == "none" else s["param"].to(DTYPES[case["copy"]])
    s["grad_scale"] = torch.tensor([0.75], dtype=torch.float32, device="cuda")     # clipping by the global norm
    return s


_context = {}


def _library():
    """The package and its context on this device, made once as a program does at its start."""
    if not _context:
        import paper_2605_26660_b200 as wq
        _context["wq"], _context["ctx"] = wq, wq.windq_create()
    return _context["wq"], _context["ctx"]


def prepare(case, seed):
    if case["op"] != "adamw":
        s = _lora_inputs(case, seed)
        s["op"] = case["op"]
        return s
    s = _adamw_inputs(case, seed)
    s["op"], s["state"] = "adamw", case["state"]
    if own:
        # the optimiser's list of tensors, made once when a training program builds its optimiser
        cut = lambda x, k=1: None if x is None else [x[a // k: a // k + -(-n // k)] for a, n in zip(s["first"], s["sizes"])]  # noqa: E731
        wq, _ = _library()
        if s["state"] == "q8":
            s["tensors"] = wq.AdamwTensors(cut(s["param"]), cut(s["grad"]), cut(s["m"]), cut(s["r"]),
                                           m_scale=cut(s["m_scale"], BLOCK), r_scale=cut(s["r_scale"], BLOCK), copies=cut(s["copy"]))
            s["values"] = (cut(s["m_value"]), cut(s["v_value"]))
            s["m_value"].zero_()
            s["v_value"].zero_()
        else:
            s["tensors"] = wq.AdamwTensors(cut(s["param"]), cut(s["grad"]), cut(s["m"]), cut(s["v"]), copies=cut(s["copy"]))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------

def _low_rank(s, x, a):
    """scaling[a] x A_a^T of every token in its own adapter's columns of [T, adapters * rank], zeros elsewhere."""
    n, r, _ = a.shape
    mine = s["adapter_of"][:, None] == torch.arange(n, device="cuda", dtype=torch.int32)[None, :]
    u = (x @ a.reshape(n * r, -1).T).view(-1, n, r) * (mine * s["scaling"])[:, :, None]
    return u.view(-1, n * r)


def _plain_lora(s):
    dt = s["X"].dtype
    x, w, a, b = (s[k].float() for k in ("X", "W", "A", "B"))
    n, r, C = a.shape
    R = b.shape[1]
    b_cols = b.permute(1, 0, 2).reshape(R, n * r)
    u = _low_rank(s, x, a)
    if s["op"] == "lora_forward":
        return {"y": (x @ w.T + u @ b_cols.T).to(dt)}
    dy = s["dY"].float()
    v = _low_rank(s, dy, b.permute(0, 2, 1))
    return {"dx": (dy @ w + v @ a.reshape(n * r, C)).to(dt), "dA": (v.T @ x).view(n, r, C),
            "dB": (dy.T @ u).view(R, n, r).permute(1, 0, 2).contiguous()}


def _own_lora(s):
    wq, ctx = _library()
    if s["op"] == "lora_forward":
        return {"y": wq.windq_lora_forward(ctx, s["X"], s["W"], s["A"], s["B"], s["scaling"], s["adapter_of"])}
    return wq.windq_lora_backward(ctx, s["X"], s["W"], s["A"], s["B"], s["scaling"], s["adapter_of"], s["dY"])


def _plain_adamw(s):
    t = s["step"]
    s["step"] = t + 1
    g = s["grad"].float() * s["grad_scale"]
    q8 = s["state"] == "q8"
    m = _decode(s["m"], s["m_scale"], 127) if q8 else s["m"]
    v = _decode(s["r"], s["r_scale"], 255).square_() if q8 else s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    r = v.sqrt()
    change = (m * (LR / (1.0 - BETA1 ** t))) / (r * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS)
    s["param"].mul_(1.0 - LR * DECAY).sub_(change)
    out = {"param": s["param"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"].copy_(s["param"])
    if q8:
        (s["m"], s["m_scale"]), (s["r"], s["r_scale"]) = _encode(m, 127, True), _encode(r, 255, False)
        return out | {"m": _decode(s["m"], s["m_scale"], 127), "v": _decode(s["r"], s["r_scale"], 255).square_()}
    s["m"], s["v"] = m, v
    return out | {"m": m, "v": v}


def _own_adamw(s):
    wq, ctx = _library()
    wq.windq_adamw_step(ctx, s["tensors"], step=s["step"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                        grad_scale=s["grad_scale"])
    s["step"] += 1
    out = {"param": s["param"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    if s["state"] == "q8":
        wq.windq_adamw_states(ctx, s["tensors"], *s["values"])
        return out | {"m": s["m_value"], "v": s["v_value"]}
    return out | {"m": s["m"], "v": s["v"]}


def run(state):
    if state["op"] == "adamw":
        return _own_adamw(state) if own else _plain_adamw(state)
    return _own_lora(state) if own else _plain_lora(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n = float(sum(_shapes(case)))
        size = {"f32": 4, "f16": 2, "bf16": 2, "none": 0}
        # parameter read and written, gradient read, states read and written, the 16-bit copy written; with 8-bit
        # states their values written out as well, since a pass returns them
        state = 16 if case["state"] == "f32" else 4 + 16.0 / BLOCK + 8
        return {"bytes": n * (8 + size[case["grad"]] + state + size[case["copy"]]), "flops": n * 16}
    T, R, C, r = (float(case[k]) for k in ("T", "R", "C", "rank"))
    used = float(min(case["adapters"], case["requests"]))
    inputs = 2 * (T * C + R * C + used * r * (R + C)) + 4 * T
    if case["op"] == "lora_forward":
        return {"bytes": inputs + 2 * T * R, "flops": 2 * T * R * C + 2 * T * r * (R + C)}
    return {"bytes": inputs + 2 * T * R + 2 * T * C + 4 * case["adapters"] * r * (R + C),
            "flops": 2 * T * R * C + 2 * T * r * (3 * C + 2 * R)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _exact_lora(case, seed):
    s = _lora_inputs(case, seed)
    x, w = s["X"].double(), s["W"].double()
    out = x @ w.T if case["op"] == "lora_forward" else s["dY"].double() @ w
    dA, dB = torch.zeros(s["A"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["B"].shape, dtype=torch.float64, device="cuda")
    for k in range(case["adapters"]):
        rows = torch.nonzero(s["adapter_of"] == k).flatten()
        if not rows.numel():
            continue
        a, b, c = s["A"][k].double(), s["B"][k].double(), s["scaling"][k].double()
        low = c * (x[rows] @ a.T)
        if case["op"] == "lora_forward":
            out[rows] += low @ b.T
            continue
        dy = s["dY"][rows].double()
        back = c * (dy @ b)
        out[rows] += back @ a
        dA[k], dB[k] = back.T @ x[rows], dy.T @ low
    return {"y": out} if case["op"] == "lora_forward" else {"dx": out, "dA": dA, "dB": dB}


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    g = s["grad"].double() * s["grad_scale"].double()
    if case["state"] == "q8":
        per = lambda x: torch.repeat_interleave(x.double(), BLOCK)  # noqa: E731
        c = s["m"].double() / 127
        m, v = c * c.abs() * per(s["m_scale"]), ((s["r"].double() / 255) ** 2 * per(s["r_scale"])) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
    mean, rms = m / (1 - BETA1 ** s["step"]), (v / (1 - BETA2 ** s["step"])).sqrt()
    p = s["param"].double() * (1 - LR * DECAY) - LR * mean / (rms + EPS)
    out = {"param": p, "m": m, "v": v}
    if case["state"] == "q8":
        out["m"] = out["v"] = None                 # codes are a choice of rounding, no value of the definition
    return out | ({} if s["copy"] is None else {"copy": p})


def exact(case, seed):
    return _exact_adamw(case, seed) if case["op"] == "adamw" else _exact_lora(case, seed)
