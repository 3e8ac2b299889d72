"""The operators of the tensor-parallel feed-forward block, as they are measured.

Four operators, each in a plain form (elementary torch operations in 32 bits, rounded once at
the end) and, where ``own`` is true, as the calls a user makes of this package:

  quantize  16-bit rows -> microscaled 4-bit floating point -> read back
  linear    a product with 4-bit weights: the activations are quantised in the call
  gated     act(x Wg^T) * (x Wu^T) over 4-bit weights
  ff        the same block over 16-bit weights, alone or as a training step with its gradients

The sizes are those of a feed-forward block split over 8 ranks whose hidden size is 3840 or 5376
(the [tokens x hidden] activations that the AllReduce of this repository reduces): a width of
4 * hidden / 8 = 1920 or 2688 for each rank, and 1 to 8192 tokens.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def listed():
    return [
        # activations of a decoding batch, on their way into a 4-bit product
        dict(name="quantize-mx-64x5376", op="quantize", format="mx", dtype="bf16", tokens=64, k=5376, pad=0),
        # odd sizes, rows inside a wider buffer (a slice of a fused projection)
        dict(name="quantize-mx-777x1250-strided", op="quantize", format="mx", dtype="fp16", tokens=777, k=1250, pad=46),
        # the activations of a long prompt
        dict(name="quantize-nv-8192x5376", op="quantize", format="nv", dtype="bf16", tokens=8192, k=5376, pad=0),
        # down projection of one decoded token on one rank
        dict(name="linear-nv-1x2688-5376", op="linear", format="nv", dtype="bf16", tokens=1, k=2688, n=5376, pad=0),
        # ragged everything: a short prompt, sizes that fill no tile
        dict(name="linear-mx-333x1000-1250", op="linear", format="mx", dtype="fp16", tokens=333, k=1000, n=1250, pad=0),
        # down projection of a long prompt on one rank
        dict(name="linear-nv-8192x2688-5376", op="linear", format="nv", dtype="bf16", tokens=8192, k=2688, n=5376, pad=0),
        # first half of the block: one decoded token, and a 2048-token prompt
        dict(name="gated-mx-1x5376-2688", op="gated", format="mx", dtype="bf16", act="gelu", tokens=1, k=5376, f=2688, pad=0),
        dict(name="gated-nv-2048x3840-1920", op="gated", format="nv", dtype="bf16", act="gelu", tokens=2048, k=3840, f=1920,
             pad=0),
        # the block with 16-bit weights: a small decoding batch (no gradients kept)
        dict(name="ff-serve-4x3840-1920", op="ff", dtype="bf16", act="gelu", tokens=4, k=3840, f=1920, pad=0, train=False),
        # training steps (forward, then all gradients): odd sizes, an ordinary step, a long one
        dict(name="ff-train-501x1000-700", op="ff", dtype="fp16", act="silu", tokens=501, k=1000, f=700, pad=0, train=True),
        dict(name="ff-train-2048x3840-1920", op="ff", dtype="bf16", act="gelu", tokens=2048, k=3840, f=1920, pad=0, train=True),
        dict(name="ff-train-8192x5376-2688", op="ff", dtype="bf16", act="gelu", tokens=8192, k=5376, f=2688, pad=0, train=True),
    ]


def _spread(rng, lo, hi, step=1):
    """a whole number of [lo, hi], uniform in its logarithm, a multiple of step"""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(step, int(v) // step * step))


def draw(rng):
    op = rng.choice(("quantize", "linear", "gated", "ff"))
    # two of three sizes are multiples of 64, as models have them; the others are what comes
    step = rng.choice((64, 64, 1))
    # tokens: a decoding batch or a prompt
    tokens = _spread(rng, 1, 8192) if rng.random() < 0.7 else rng.choice((1, 2, 4, 8, 16, 32))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "fp16")), tokens=tokens,
                pad=rng.choice((0, 0, 0, 8, 64, 13)))
    if op != "ff":
        case["format"] = rng.choice(("mx", "nv"))
    if op == "quantize":
        case["k"] = _spread(rng, 256, 5376, step)
    elif op == "linear":
        case["k"] = _spread(rng, 256, 5376, step)
        case["n"] = _spread(rng, 256, 5376, step)
    else:
        case["k"] = _spread(rng, 256, 5376, step)
        case["f"] = _spread(rng, 128, 2688, step)
        case["act"] = rng.choice(("gelu", "silu"))
    if op == "ff":
        case["train"] = rng.random() < 0.7
    return case


def work(case):
    m, k = case["tokens"], case["k"]
    op = case["op"]
    # bytes of one quantised element: 4 bits, and its share of the block's and the row's scale
    four = lambda rows, cols: (rows * cols / 2 + rows * (-(-cols // 32))) if case["format"] == "mx" else \
        (rows * cols / 2 + rows * (-(-cols // 16)) + 4 * rows)
    if op == "quantize":
        return {"bytes": 2 * m * k + 2 * four(m, k) + 2 * m * k, "flops": 4 * m * k}
    if op == "linear":
        n = case["n"]
        return {"bytes": 2 * m * k + four(n, k) + 2 * m * n, "flops": 2 * m * n * k}
    f = case["f"]
    if op == "gated":
        return {"bytes": 2 * m * k + 2 * four(f, k) + 2 * m * f, "flops": 4 * m * f * k}
    if not case["train"]:
        return {"bytes": 2 * (m * k + 2 * f * k + m * f), "flops": 4 * m * f * k}
    # x, dh, both weights in; h, dx, both weights' gradients out
    return {"bytes": 2 * (m * k + m * f + 2 * f * k) + 2 * (m * f + m * k + 2 * f * k), "flops": 12 * m * f * k}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _inputs(case, seed):
    """16-bit tensors of the case, from the seed alone"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    m, k = case["tokens"], case["k"]

    def normal(rows, cols, scale):
        return (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dtype)

    wide = torch.randn(m, k + case["pad"], generator=gen, device="cuda")
    if case["op"] != "ff":
        # outlier channels, as activations have them: 1 in 100, fifty times as large
        hot = torch.randperm(k, generator=gen, device="cuda")[:max(1, k // 100)]
        wide[:, hot] *= 50.0
    data = {"x": wide.to(dtype)[:, :k]}
    if case["op"] == "linear":
        data["w"] = normal(case["n"], k, k ** -0.5)
    elif case["op"] in ("gated", "ff"):
        data["wg"] = normal(case["f"], k, k ** -0.5)
        data["wu"] = normal(case["f"], k, k ** -0.5)
        if case["op"] == "ff" and case["train"]:
            data["dh"] = normal(m, case["f"], 1.0)
    return data


def prepare(case, seed):
    state = dict(case)
    data = _inputs(case, seed)
    weights = {"linear": ("w",), "gated": ("wg", "wu")}.get(case["op"], ())
    if own:
        from paper_2506_17615_b200 import feedforward
        state["ff"] = feedforward
        state["format_id"] = {"mx": feedforward.FP4_MX, "nv": feedforward.FP4_NV}.get(case.get("format"))
        state["act_id"] = {"gelu": feedforward.ACT_GELU_TANH, "silu": feedforward.ACT_SILU}.get(case.get("act"))
        for name in weights:        # a serving program quantises its weights once
            data[name] = feedforward.fp4_quantize(data[name], state["format_id"])
    else:
        for name in weights:
            data[name] = _plain_quantize(data[name].float(), case["format"])
    state.update(data)
    return state


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------

def _blocks(x, block):
    rows, cols = x.shape
    whole = -(-cols // block) * block
    if whole != cols:
        x = torch.cat([x, x.new_zeros(rows, whole - cols)], dim=1)
    return x.reshape(rows, whole // block, block)


def _plain_e2m1(y):
    """nearest 4-bit code (a signed index into E2M1's magnitudes), ties to the even index"""
    a = y.abs()
    index = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + \
        (a >= 3.5).int() + (a > 5.0).int()
    return torch.where(y < 0, -index, index).to(torch.int8)


def _plain_quantize(x, fmt):
    """codes [rows, blocks, block], what multiplies them [rows, blocks], and the number of columns"""
    if fmt == "mx":
        v = _blocks(x, 32)
        amax = v.abs().amax(dim=2)
        exponent = torch.clamp(torch.frexp(amax)[1] - 3, min=-127)        # floor(log2(amax)) - 2
        exponent = torch.where(amax > 0, exponent, torch.full_like(exponent, -127))
        one = torch.ones_like(amax)
        scale = torch.ldexp(torch.ldexp(one, exponent // 2), exponent - exponent // 2)
        inverse = torch.ldexp(torch.ldexp(one, -(exponent // 2)), exponent // 2 - exponent)
        return _plain_e2m1(v * inverse[:, :, None]), scale, x.shape[1]
    v = _blocks(x, 16)
    amax = v.abs().amax(dim=2)
    top = amax.amax(dim=1, keepdim=True)
    live = top >= 2.0 ** -100
    safe = torch.where(live, top, torch.ones_like(top))
    row = torch.div(safe, torch.full_like(safe, 2688.0))
    up = torch.div(torch.full_like(safe, 448.0), safe)
    s = torch.clamp(amax * up, max=448.0).to(torch.float8_e4m3fn).float()
    s = torch.where(live, s, torch.zeros_like(s))
    d = s * row
    inverse = torch.where(s > 0, torch.div(torch.ones_like(d), torch.where(s > 0, d, torch.ones_like(d))), torch.zeros_like(d))
    return _plain_e2m1(v * inverse[:, :, None]), d, x.shape[1]


def _plain_values(q):
    codes, scale, cols = q
    table = torch.tensor(E2M1, device=codes.device)
    index = codes.int()
    v = table[index.abs().long()] * torch.sign(index).float() * scale[:, :, None]
    return v.reshape(codes.shape[0], -1)[:, :cols]


def _plain_act(g, act):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)


def _run_plain(s):
    x, dtype = s["x"].float(), s["x"].dtype
    if s["op"] == "quantize":
        return _plain_values(_plain_quantize(x, s["format"])).to(dtype)
    if s["op"] == "linear":
        xq = _plain_values(_plain_quantize(x, s["format"]))
        return (xq @ _plain_values(s["w"]).t()).to(dtype)
    if s["op"] == "gated":
        xq = _plain_values(_plain_quantize(x, s["format"]))
        g, u = xq @ _plain_values(s["wg"]).t(), xq @ _plain_values(s["wu"]).t()
        return (_plain_act(g, s["act"])[0] * u).to(dtype)
    wg, wu = s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _plain_act(g, s["act"])
    h = (a * u).to(dtype)
    if not s["train"]:
        return h
    dh = s["dh"].float()
    du, dg = dh * a, dh * u * slope
    return {"h": h, "dx": (dg @ wg + du @ wu).to(dtype), "dwg": (dg.t() @ x).to(dtype), "dwu": (du.t() @ x).to(dtype)}


def _run_own(s):
    ff = s["ff"]
    if s["op"] == "quantize":
        return ff.fp4_dequantize(ff.fp4_quantize(s["x"], s["format_id"]), s["x"].dtype)
    if s["op"] == "linear":
        return ff.fp4_linear(s["x"], s["w"])
    if s["op"] == "gated":
        return ff.fp4_gated(s["x"], s["wg"], s["wu"], s["act_id"])
    if not s["train"]:
        return ff.gated_forward(s["x"], s["wg"], s["wu"], s["act_id"])
    h, g, u = ff.gated_forward(s["x"], s["wg"], s["wu"], s["act_id"], save=True)
    dx, dwg, dwu = ff.gated_backward(s["dh"], s["x"], s["wg"], s["wu"], g, u, s["act_id"])
    return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------

def _single(t):
    """a 64-bit value rounded to 32 bits where the definition says so"""
    return t.float().double()


def _grid(y, smallest, digits, top):
    """y >= 0 to the nearest number of `digits` binary digits whose step is at least `smallest`"""
    exponent = torch.floor(torch.log2(torch.clamp(y, min=1e-300)))
    exponent = torch.where(torch.exp2(exponent) > y, exponent - 1, exponent)
    step = torch.clamp(torch.exp2(exponent - (digits - 1)), min=smallest)
    return torch.clamp(torch.round(y / step) * step, max=top)


def _exact_values(x, fmt):
    rows, cols = x.shape
    size = 32 if fmt == "mx" else 16
    count = -(-cols // size)
    v = torch.zeros(rows, count * size, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, count, size)
    peak = v.abs().amax(2, keepdim=True)
    if fmt == "mx":
        mantissa, power = np.frexp(peak.cpu().numpy())
        power = torch.from_numpy(np.where(mantissa > 0, np.maximum(power - 3, -127), -127)).to(x.device)
        d = torch.exp2(power.double())
        y = v / d
    else:
        top = peak.amax(1, keepdim=True)
        dead = top < 2.0 ** -100
        top = torch.where(dead, torch.ones_like(top), top)
        s = _grid(torch.clamp(_single(peak * _single(448.0 / top)), max=448.0), 2.0 ** -9, 4, 448.0)
        s = torch.where(dead, torch.zeros_like(s), s)
        d = _single(s * _single(top / 2688.0))
        y = torch.where(s > 0, _single(v * _single(1.0 / torch.where(s > 0, d, torch.ones_like(d)))), torch.zeros_like(v))
    q = torch.copysign(_grid(y.abs(), 0.5, 2, 6.0), y)
    return (q * d).view(rows, -1)[:, :cols]


def _exact_act(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    z = math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
    s = torch.sigmoid(z)
    return g * s, s + g * s * (1 - s) * math.sqrt(8.0 / math.pi) * (1 + 0.134145 * g ** 2)


def exact(case, seed):
    data = {name: t.double() for name, t in _inputs(case, seed).items()}
    op = case["op"]
    if op == "ff":
        x, wg, wu = data["x"], data["wg"], data["wu"]
        g, u = x @ wg.T, x @ wu.T
        a, slope = _exact_act(g, case["act"])
        if not case["train"]:
            return a * u
        du = data["dh"] * a
        dg = data["dh"] * u * slope
        return {"h": a * u, "dx": dg @ wg + du @ wu, "dwg": dg.T @ x, "dwu": du.T @ x}
    x = _exact_values(data["x"], case["format"])
    if op == "quantize":
        return x
    if op == "linear":
        return x @ _exact_values(data["w"], case["format"]).T
    return _exact_act(x @ _exact_values(data["wg"], case["format"]).T, case["act"])[0] * \
        (x @ _exact_values(data["wu"], case["format"]).T)
