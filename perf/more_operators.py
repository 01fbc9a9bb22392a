"""Cases and plain forms of the operators of a quantised model's feed-forward block: trained in 16 bits, served in 8.

Five operators, each through the package's public calls where ``own`` is set and in elementary torch operations in
32 bits (integer sums and positions next to a rounding border in 64) where it is not:

  quantize_rows   q[t][j] = round(127 x[t][j] / a[t]), a[t] = max_j |x[t][j]|, scale[t] = a[t] / 127; a pass returns the
                  values q scale, in the type of x, and the scales
  int8_forward    Y[t][r] = scale_x[t] scale_w[r] sum_j qx[t][j] qw[r][j]: a pass takes tokens of 16 bits, quantises them
                  and multiplies them with weights that were quantised when the model was loaded
  gated_forward   H = act(X Wg^T) * (X Wu^T), and, where a backward pass follows, both products
  gated_int8      the same from 8-bit codes of the weights, tokens quantised within the pass as in int8_forward
  gated_backward  dX, dWg, dWu from dH and the two products that the forward pass kept

act is silu, g / (1 + exp(-g)), or the tanh form of gelu, g / (1 + exp(-2 sqrt(2 / pi) (g + 0.044715 g^3))).
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
GELU_A, GELU_B = 2.0 * math.sqrt(2.0 / math.pi), 0.044715


def _case(op, name, T, out, C, dtype, act="none", saved=False):
    """T tokens of C channels; `out` outputs (gated operators: the width of H; quantize_rows: none)."""
    return {"name": name, "op": op, "T": T, "out": out, "C": C, "dtype": dtype, "act": act, "saved": saved}


def listed():
    return [
        # one token before the first projection of a 1B-shaped model: launch latency
        _case("quantize_rows", "quantize_one_token", 1, 0, 2048, "f16"),
        # the down projection of an 8B-shaped model, quantised row by row when it is loaded: memory
        _case("quantize_rows", "quantize_down_weight", 4096, 0, 14336, "bf16"),
        # one user, one token, the query projection of a 1B-shaped model: latency
        _case("int8_forward", "int8_one_token", 1, 2048, 2048, "f16"),
        # a batch of requests, the down projection of a 7B-shaped model: the bytes of the weight
        _case("int8_forward", "int8_48_requests", 48, 4096, 11008, "bf16"),
        # long prompts, the gate projection of an 8B-shaped model: tensor cores
        _case("int8_forward", "int8_prompts_long", 8192, 14336, 4096, "bf16"),
        # one token through the block of a 1B-shaped model
        _case("gated_forward", "gated_one_token", 1, 8192, 2048, "f16", "silu"),
        # a few prompts packed without padding, a 13B-shaped block, a width that ends inside every tile
        _case("gated_forward", "gated_prompts_ragged", 777, 13821, 5120, "bf16", "gelu"),
        # a training batch of a 7B-shaped block, with what the backward pass needs
        _case("gated_forward", "gated_training", 4096, 11008, 4096, "bf16", "silu", True),
        # 33 requests through a 7B-shaped block in 8 bits: the bytes of the weights
        _case("gated_int8", "gated_int8_33_requests", 33, 11008, 4096, "f16", "silu"),
        # prompts through an 8B-shaped block in 8 bits
        _case("gated_int8", "gated_int8_prompts", 2048, 14336, 4096, "bf16", "silu"),
        # one short sequence, a 1B-shaped block, odd lengths
        _case("gated_backward", "gated_backward_short", 333, 8191, 2048, "f16", "gelu"),
        # the training batch
        _case("gated_backward", "gated_backward_training", 4096, 11008, 4096, "bf16", "silu"),
    ]


def _log_int(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


# products T * out * C of the largest listed case of every operator
LARGEST = {"quantize_rows": 4096 * 14336, "int8_forward": 8192 * 14336 * 4096, "gated_forward": 4096 * 11008 * 4096,
           "gated_int8": 2048 * 14336 * 4096, "gated_backward": 4096 * 11008 * 4096}


def draw(rng):
    op = rng.choice(["quantize_rows", "int8_forward", "int8_forward", "gated_forward", "gated_int8", "gated_backward"])
    T, out, C = _log_int(rng, 1, 8192), _log_int(rng, 256, 14336), _log_int(rng, 256, 14336)
    if rng.random() < 0.6:                      # widths of models are round, most of the time
        out, C = out + -out % 64, C + -C % 64
    if op == "quantize_rows":
        out = 0
    while T * max(out, 1) * C > LARGEST[op] or out * C > 14336 * 4096:
        T, out, C = max(1, T * 7 // 8), out * 15 // 16, C * 15 // 16
    return {"op": op, "T": T, "out": out, "C": C, "dtype": rng.choice(["f16", "bf16"]),
            "act": rng.choice(["silu", "gelu"]) if op.startswith("gated") else "none",
            "saved": op == "gated_forward" and rng.random() < 0.5}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(x, dtype, step):
    """x in `dtype`, its rows `step` elements apart or a multiple of that, as the calls take them."""
    T, C = x.shape
    return torch.empty((T, C + -C % step), dtype=dtype, device=x.device)[:, :C].copy_(x)


def _tokens(case, g):
    T, C = case["T"], case["C"]
    x = _randn((T, C), g) * (0.5 * _randn((C,), g)).exp_()        # channels of unequal scale ...
    x[:, torch.randint(0, C, (4,), generator=g, device="cuda")] *= 20.0          # ... and a few hot ones
    return _rows(x, DTYPES[case["dtype"]], 8)


def _weight(case, g):
    step = 0.005 + 0.005 * torch.rand((case["out"], 1), generator=g, device="cuda")   # a quantised weight: few levels a row
    w = _randn((case["out"], case["C"]), g).mul_(0.02).div_(step).round_().mul_(step)
    return _rows(w, DTYPES[case["dtype"]], 8)


def _codes(x):
    """Codes and scales of rows that hold a 16-bit type: 127 x and, for such x, the quotient's side of every border between
    two codes are exact in 32 bits."""
    x = x.float()
    a = x.abs().amax(dim=1)
    return torch.round(x * 127.0 / a.clamp(min=1e-30)[:, None]), a / 127.0


def _coded_weight(case, g):
    q, scale = _codes(_weight(case, g))
    return _rows(q, torch.int8, 16), scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "quantize_rows":
        return {"X": _weight(case | {"out": case["T"]}, g) if case["T"] > 1 else _tokens(case, g)}
    s = {"X": _tokens(case, g)}
    if op == "int8_forward":
        s["W"] = _coded_weight(case, g)
    elif op == "gated_int8":
        s["Wg"], s["Wu"] = _coded_weight(case, g), _coded_weight(case, g)
    else:
        s["Wg"], s["Wu"] = _weight(case, g), _weight(case, g)
    if op == "gated_backward":
        # what the forward pass of the same step left
        s["gate"], s["up"] = _rows(s["X"] @ s["Wg"].T, dt, 8), _rows(s["X"] @ s["Wu"].T, dt, 8)
        size = 0.01 * (0.5 * _randn((case["T"], 1), g)).exp_()        # tokens of unequal weight in the loss
        s["dH"] = _rows(_randn((case["T"], case["out"]), g) * size, dt, 8)
    return s


_context = {}


def _library():
    """The package and its context on this device, made once as a program does at its start."""
    if not _context:
        import paper_2605_26660_b200 as wq
        _context["wq"], _context["ctx"] = wq, wq.windq_create()
    return _context["wq"], _context["ctx"]


def prepare(case, seed):
    return _inputs(case, seed) | {"op": case["op"], "act": case["act"], "saved": case["saved"], "dtype": DTYPES[case["dtype"]]}


# ---- one pass --------------------------------------------------------------------------------------------------

def _exponent(g, act):
    return g if act == "silu" else GELU_A * (g + GELU_B * g ** 3)


def _gate(g, act):
    return g / (1.0 + torch.exp(-_exponent(g, act)))


def _integer_product(x, w):
    q, sx = _codes(x)
    return (q.double() @ w[0].T.double()).float() * sx[:, None] * w[1][None, :]


def _plain(s):
    op, dt, act = s["op"], s["dtype"], s["act"]
    if op == "quantize_rows":
        q, scale = _codes(s["X"])
        return {"values": (q * scale[:, None]).to(dt), "scale": scale}
    if op == "int8_forward":
        return {"y": _integer_product(s["X"], s["W"]).to(dt)}
    if op == "gated_int8":
        return {"h": (_gate(_integer_product(s["X"], s["Wg"]), act) * _integer_product(s["X"], s["Wu"])).to(dt)}
    x, wg, wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
    if op == "gated_forward":
        g, u = x @ wg.T, x @ wu.T
        out = {"h": (_gate(g, act) * u).to(dt)}
        return out | {"gate": g.to(dt), "up": u.to(dt)} if s["saved"] else out
    g, u, dh = s["gate"].float(), s["up"].float(), s["dH"].float()
    p = 1.0 / (1.0 + torch.exp(-_exponent(g, act)))
    slope = 1.0 if act == "silu" else GELU_A * (1.0 + 3.0 * GELU_B * g * g)
    du = dh * g * p
    dg = dh * u * (p + g * p * (1.0 - p) * slope)
    return {"dx": (dg @ wg + du @ wu).to(dt), "dWg": (dg.T @ x).to(dt), "dWu": (du.T @ x).to(dt)}


def _own(s):
    wq, ctx = _library()
    op = s["op"]
    if op == "quantize_rows":
        r = wq.windq_quantize_rows(ctx, s["X"], want_values=True)
        return {"values": r["values"], "scale": r["scale"]}
    if op == "int8_forward":
        q = wq.windq_quantize_rows(ctx, s["X"])
        return {"y": wq.windq_int8_forward(ctx, q["codes"], q["scale"], *s["W"], dtype=s["dtype"])}
    if op == "gated_int8":
        q = wq.windq_quantize_rows(ctx, s["X"])
        return {"h": wq.windq_gated_int8_forward(ctx, q["codes"], q["scale"], *s["Wg"], *s["Wu"], activation=s["act"],
                                                 dtype=s["dtype"])}
    if op == "gated_forward":
        r = wq.windq_gated_forward(ctx, s["X"], s["Wg"], s["Wu"], activation=s["act"], want_saved=s["saved"])
        return r if s["saved"] else {"h": r["h"]}
    return wq.windq_gated_backward(ctx, s["X"], s["Wg"], s["Wu"], s["dH"], gate=s["gate"], up=s["up"], activation=s["act"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    op, T, F, C = case["op"], float(case["T"]), float(case["out"]), float(case["C"])
    if op == "quantize_rows":
        return {"bytes": 2 * T * C + T * C * 2 + 4 * T, "flops": 4 * T * C}
    if op == "int8_forward":
        return {"bytes": 2 * T * C + F * C + 4 * F + 2 * T * F, "flops": 2 * T * F * C}
    if op == "gated_int8":
        return {"bytes": 2 * T * C + 2 * F * C + 8 * F + 2 * T * F, "flops": 4 * T * F * C}
    if op == "gated_forward":
        return {"bytes": 2 * T * C + 4 * F * C + 2 * T * F * (3 if case["saved"] else 1), "flops": 4 * T * F * C}
    return {"bytes": 2 * T * C + 4 * F * C + 6 * T * F + 2 * T * C + 4 * F * C, "flops": 8 * T * F * C}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _exact_codes(x):
    x = x.double()
    top = x.abs().max(dim=1, keepdim=True).values
    return (127 * x / top.clamp(min=1e-300)).round(), top / 127


def _exact_activation(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g.pow(3))))


def _exact_slope(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return s + g * s * (1 - s)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g.pow(3)))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t.square()) * k * (1 + 3 * 0.044715 * g.square())


def exact(case, seed):
    s, op, act = _inputs(case, seed), case["op"], case["act"]
    if op == "quantize_rows":
        q, scale = _exact_codes(s["X"])
        return {"values": q * scale, "scale": scale[:, 0]}
    if op in ("int8_forward", "gated_int8"):
        q, scale = _exact_codes(s["X"])
        x = q * scale
        value = lambda w: w[0].double() * w[1].double()[:, None]  # noqa: E731
        if op == "int8_forward":
            return {"y": x @ value(s["W"]).T}
        return {"h": _exact_activation(x @ value(s["Wg"]).T, act) * (x @ value(s["Wu"]).T)}
    x, wg, wu = s["X"].double(), s["Wg"].double(), s["Wu"].double()
    if op == "gated_forward":
        g, u = x @ wg.T, x @ wu.T
        out = {"h": _exact_activation(g, act) * u}
        return out | {"gate": g, "up": u} if case["saved"] else out
    g, u, dh = s["gate"].double(), s["up"].double(), s["dH"].double()
    du, dg = dh * _exact_activation(g, act), dh * u * _exact_slope(g, act)
    return {"dx": dg @ wg + du @ wu, "dWg": dg.T @ x, "dWu": du.T @ x}
