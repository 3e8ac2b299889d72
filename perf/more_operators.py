"""Operators beside the feed-forward block, as they are measured.

Each in a plain form (elementary torch operations in 32 bits, rounded once at the end) and, where ``own`` is
true, as the calls a user makes of this package:

  norm      residual addition and root-mean-square norm, alone (serving) or with all gradients (a training step)
  norm8     the same norm, its output in 8 bits (E4M3 elements, a power of two for each 32 of a row), and these read back
  product8  products of matrices in that form: x w^T with x quantised in the call, or the gated block
            act(x Wg^T) * (x Wu^T) over the norm's 8-bit output
  adapters  out = y + c (x A^T) B^T, every token with the low-rank adapter of its own request

They stand between one AllReduce of this repository and the next block's projections, so the sizes are those of
perf/operators.py: hidden sizes 3840 and 5376 (rows of the tensors that are reduced), a block's width of 1920 or 2688 on each of
8 ranks, 1 to 8192 tokens.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoded token between an AllReduce and the next 16-bit projection: latency is all there is
        dict(name="norm-1x3840", op="norm", dtype="bf16", wtype="bf16", tokens=1, k=3840, pad=0, offset=1.0, train=False),
        # training steps: odd sizes with the weight kept in fp32, and the rows of a long batch
        dict(name="norm-train-501x1000", op="norm", dtype="fp16", wtype="fp32", tokens=501, k=1000, pad=0, offset=0.0, train=True),
        dict(name="norm-train-8192x5376", op="norm", dtype="bf16", wtype="bf16", tokens=8192, k=5376, pad=0, offset=1.0,
             train=True),
        # a decoding batch on its way into an 8-bit projection
        dict(name="norm8-64x5376", op="norm8", dtype="bf16", wtype="bf16", tokens=64, k=5376, pad=0, offset=1.0),
        # a short prompt, odd sizes, rows inside a wider buffer
        dict(name="norm8-777x1250-strided", op="norm8", dtype="fp16", wtype="fp16", tokens=777, k=1250, pad=46, offset=0.0),
        # a long prompt
        dict(name="norm8-8192x5376", op="norm8", dtype="bf16", wtype="bf16", tokens=8192, k=5376, pad=0, offset=1.0),
        # the block's first half for one decoded token, from the norm's 8-bit output
        dict(name="product8-gated-1x5376-2688", op="product8", form="gated", dtype="bf16", act="gelu", tokens=1, k=5376, n=2688,
             pad=0),
        # ragged everything: a short prompt's 16-bit activations, sizes that fill no tile
        dict(name="product8-linear-333x1000-1250", op="product8", form="linear", dtype="fp16", act="", tokens=333, k=1000, n=1250,
             pad=0),
        # the block's first half for a long prompt
        dict(name="product8-gated-8192x5376-2688", op="product8", form="gated", dtype="bf16", act="gelu", tokens=8192, k=5376,
             n=2688, pad=0),
        # one decoded token with its adapter beside the down projection of a rank
        dict(name="adapters-1x2688-5376", op="adapters", dtype="bf16", tokens=1, k=2688, n=5376, rank=16, requests=1, pad=0),
        # a decoding batch: 64 requests, each with an adapter of its own
        dict(name="adapters-64x2688-5376", op="adapters", dtype="bf16", tokens=64, k=2688, n=5376, rank=16, requests=64, pad=0),
        # prompts of seven requests in one batch, of ragged lengths, the last one without an adapter
        dict(name="adapters-8192x2688-5376", op="adapters", dtype="bf16", tokens=8192, k=2688, n=5376, rank=64, requests=7, pad=0),
    ]


def _spread(rng, lo, hi, step=1):
    """a whole number of [lo, hi], uniform in its logarithm, a multiple of step"""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(step, int(v) // step * step))


def draw(rng):
    op = rng.choice(("norm", "norm8", "product8", "adapters"))
    # two of three sizes are multiples of 64, as models have them; the others are what comes
    step = rng.choice((64, 64, 1))
    # tokens: a decoding batch or a prompt
    tokens = _spread(rng, 1, 8192) if rng.random() < 0.7 else rng.choice((1, 2, 4, 8, 16, 32, 64))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "fp16")), tokens=tokens, pad=rng.choice((0, 0, 0, 8, 64, 13)))
    if op in ("norm", "norm8"):
        case["k"] = _spread(rng, 64, 5376, step)
        case["wtype"] = rng.choice((case["dtype"], case["dtype"], "fp32"))
        case["offset"] = rng.choice((0.0, 1.0))
        if op == "norm":
            case["train"] = rng.random() < 0.6
    elif op == "product8":
        case["form"] = rng.choice(("linear", "gated"))
        case["k"] = _spread(rng, 256, 5376, step)
        case["n"] = _spread(rng, 128, 5376 if case["form"] == "linear" else 2688, step)
        case["act"] = rng.choice(("gelu", "silu")) if case["form"] == "gated" else ""
    else:
        case["k"] = _spread(rng, 256, 2688, step)
        case["n"] = _spread(rng, 256, 5376, step)
        case["rank"] = rng.choice((8, 16, 16, 32, 64))
        case["requests"] = tokens if tokens <= 64 else rng.choice((1, 3, 8, 20))
    return case


def _lengths(case):
    """tokens of each request, ragged; with more than one request, the last has no adapter unless each has one token"""
    m, q = case["tokens"], case["requests"]
    ends = [m if i == q else max(i, int(m * (i / q) ** 1.3)) for i in range(q + 1)]
    return [b - a for a, b in zip(ends, ends[1:])]


def _adapted(case):
    lengths = _lengths(case)
    return lengths if len(lengths) == 1 or case["tokens"] == case["requests"] else lengths[:-1]


def work(case):
    m, k, op = case["tokens"], case["k"], case["op"]
    wide = {"fp32": 4}.get(case.get("wtype"), 2)
    eight = lambda rows, cols: rows * cols + rows * (-(-cols // 32))        # a matrix in 8 bits with its scales
    if op == "norm":
        if not case["train"]:
            return {"bytes": 8 * m * k + wide * k, "flops": 6 * m * k}      # x, residual in; sum, y out
        # and dy, the sum's own gradient in; dx, dw out (the sum is read again)
        return {"bytes": 8 * m * k + 8 * m * k + 2 * wide * k, "flops": 20 * m * k}
    if op == "norm8":
        # x, residual in; sum, 8 bits out; read back: 8 bits in, their values out
        return {"bytes": 6 * m * k + 2 * eight(m, k) + 2 * m * k + wide * k, "flops": 10 * m * k}
    n = case["n"]
    if op == "product8":
        if case["form"] == "linear":
            return {"bytes": 2 * m * k + eight(n, k) + 2 * m * n, "flops": 2 * m * n * k}
        return {"bytes": eight(m, k) + 2 * eight(n, k) + 2 * m * n, "flops": 4 * m * n * k}
    used = _adapted(case)
    return {"bytes": 2 * (sum(used) * k + 2 * m * n + len(used) * case["rank"] * (k + n)),
            "flops": 2 * sum(used) * case["rank"] * (k + n)}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _inputs(case, seed):
    """tensors of the case, from the seed alone"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, op = DTYPES[case["dtype"]], case["op"]
    m, k, pad = case["tokens"], case["k"], case["pad"]

    def normal(rows, cols, scale=1.0, pad=0, type=dtype):
        return (torch.randn(rows, cols + pad, generator=gen, device="cuda") * scale).to(type)[:, :cols]

    def activations():
        # outlier channels: 1 in 100, fifty times as large
        x = torch.randn(m, k + pad, generator=gen, device="cuda")
        hot = torch.randperm(k, generator=gen, device="cuda")[:max(1, k // 100)]
        x[:, hot] *= 50.0
        return x.to(dtype)[:, :k]

    if op in ("norm", "norm8"):
        data = {"x": activations(), "residual": normal(m, k, 4.0, pad),
                "weight": (torch.randn(k, generator=gen, device="cuda") * 0.3 + (1.0 - case["offset"])).to(DTYPES[case["wtype"]])}
        if case.get("train"):
            data["dy"], data["dsum"] = normal(m, k), normal(m, k)
    elif op == "product8":
        data = {"x": activations()}
        for name in ("w",) if case["form"] == "linear" else ("wg", "wu"):
            data[name] = normal(case["n"], k, k ** -0.5)
    else:
        n, rank = case["n"], case["rank"]
        used = _adapted(case)
        data = {"x": normal(m, k, 1.0, pad), "y": normal(m, n, 1.0, pad),
                "a": normal(len(used) * rank, k, k ** -0.5).reshape(len(used), rank, k),
                "b": normal(len(used) * n, rank, rank ** -0.5).reshape(len(used), n, rank),
                "scale": torch.rand(len(used), generator=gen, device="cuda") + 0.5}
        # which adapter a request has is chance; tokens of the last request may have none
        order = torch.randperm(len(used), generator=gen, device="cuda").tolist()
        index = [i for i, length in zip(order, used) for _ in range(length)]
        data["index"] = torch.tensor(index + [-1] * (m - len(index)), dtype=torch.int32, device="cuda")
    return data


def prepare(case, seed):
    state = dict(case)
    data = _inputs(case, seed)
    # a serving program keeps its weights in 8 bits, and the gated block's input comes from the norm in 8 bits
    kept = () if case["op"] != "product8" else ("w",) if case["form"] == "linear" else ("x", "wg", "wu")
    if own:
        from paper_2506_17615_b200 import adapters, feedforward, norm
        state.update(ff=feedforward, nm=norm, ad=adapters)
        state["act_id"] = {"gelu": feedforward.ACT_GELU_TANH, "silu": feedforward.ACT_SILU}.get(case.get("act"))
        for name in kept:
            data[name] = feedforward.fp8_quantize(data[name])
    else:
        for name in kept:
            data[name] = _plain_quantize(data[name].float())
    state.update(data)
    return state


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------

def _plain_quantize(v):
    """codes' values [rows, blocks, 32], what multiplies them [rows, blocks], and the number of columns"""
    rows, cols = v.shape
    whole = -(-cols // 32) * 32
    if whole != cols:
        v = torch.cat([v, v.new_zeros(rows, whole - cols)], dim=1)
    v = v.reshape(rows, whole // 32, 32)
    amax = v.abs().amax(dim=2)
    exponent = torch.clamp(torch.frexp(amax)[1] - 9, min=-127)              # floor(log2(amax)) - 8
    exponent = torch.where(amax > 0, exponent, torch.full_like(exponent, -127))
    one = torch.ones_like(amax)
    scale = torch.ldexp(torch.ldexp(one, exponent // 2), exponent - exponent // 2)
    inverse = torch.ldexp(torch.ldexp(one, -(exponent // 2)), exponent // 2 - exponent)
    codes = torch.clamp(v * inverse[:, :, None], -448.0, 448.0).to(torch.float8_e4m3fn)
    return codes, scale, cols


def _plain_values(q):
    codes, scale, cols = q
    return (codes.float() * scale[:, :, None]).reshape(codes.shape[0], -1)[:, :cols]


def _plain_act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _plain_norm(s):
    """the sum in 16 bits and in 32, what normalises its rows, and the normalised rows times the weight.  The mean square
    is a long sum, and 8-bit outputs lie next to borders: it is taken in 64 bits."""
    total = (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    h = total.float()
    r = (1.0 / torch.sqrt(h.double().square().mean(dim=1, keepdim=True) + EPS)).float()
    return total, h, r, (h * r) * (s["weight"].float() + s["offset"])


def _run_plain(s):
    op, dtype = s["op"], s["x"][0].dtype if isinstance(s["x"], tuple) else s["x"].dtype
    if op == "norm":
        total, h, r, y = _plain_norm(s)
        if not s["train"]:
            return {"sum": total, "y": y.to(dtype)}
        n, dy = h * r, s["dy"].float()
        g = dy * (s["weight"].float() + s["offset"])
        dx = s["dsum"].float() + r * (g - n * (g * n).mean(dim=1, keepdim=True))
        return {"sum": total, "y": y.to(dtype), "dx": dx.to(dtype), "dw": (dy * n).sum(dim=0).to(s["weight"].dtype)}
    if op == "norm8":
        total, _, _, y = _plain_norm(s)
        return {"sum": total, "y": _plain_values(_plain_quantize(y)).to(dtype)}
    if op == "product8":
        if s["form"] == "linear":
            return (_plain_values(_plain_quantize(s["x"].float())) @ _plain_values(s["w"]).t()).to(dtype)
        x = _plain_values(s["x"])
        g, u = x @ _plain_values(s["wg"]).t(), x @ _plain_values(s["wu"]).t()
        return (_plain_act(g, s["act"]) * u).to(DTYPES[s["dtype"]])
    # every token against every adapter; what is not its own counts nothing
    a, b = s["a"].float(), s["b"].float()
    count, rank, k = a.shape
    mine = (s["index"][:, None] == torch.arange(count, device=a.device)[None, :]).float() * s["scale"][None, :]
    down = (s["x"].float() @ a.reshape(count * rank, k).t()).reshape(-1, count, rank) * mine[:, :, None]
    return (s["y"].float() + down.reshape(-1, count * rank) @ b.permute(0, 2, 1).reshape(count * rank, -1)).to(dtype)


def _run_own(s):
    op = s["op"]
    if op == "norm":
        if not s["train"]:
            y, total = s["nm"].add_rms_norm(s["x"], s["residual"], s["weight"], EPS, s["offset"])
            return {"sum": total, "y": y}
        y, total, factors = s["nm"].add_rms_norm(s["x"], s["residual"], s["weight"], EPS, s["offset"], save=True)
        dx, dw = s["nm"].add_rms_norm_backward(s["dy"], s["dsum"], total, factors, s["weight"], s["offset"])
        return {"sum": total, "y": y, "dx": dx, "dw": dw}
    if op == "norm8":
        q, total = s["nm"].add_rms_norm_fp8(s["x"], s["residual"], s["weight"], EPS, s["offset"])
        return {"sum": total, "y": s["ff"].fp8_dequantize(q, s["x"].dtype)}
    if op == "product8":
        if s["form"] == "linear":
            return s["ff"].fp8_linear(s["x"], s["w"])
        return s["ff"].fp8_gated(s["x"], s["wg"], s["wu"], s["act_id"], DTYPES[s["dtype"]])
    return s["ad"].add_adapters(s["y"], s["x"], s["a"], s["b"], s["index"], s["scale"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------

def _single(t):
    """a 64-bit value rounded to 32 bits where the definition says so"""
    return t.float().double()


def _exact_values(v):
    rows, cols = v.shape
    count = -(-cols // 32)
    blocks = torch.zeros(rows, count * 32, dtype=torch.float64, device=v.device)
    blocks[:, :cols] = v
    blocks = blocks.view(rows, count, 32)
    mantissa, power = np.frexp(blocks.abs().amax(2, keepdim=True).cpu().numpy())
    power = torch.from_numpy(np.where(mantissa > 0, np.maximum(power - 9, -127), -127)).to(v.device)
    d = torch.exp2(power.double())
    y = (blocks / d).abs()
    # to the nearest number of four binary digits, whose step is at least 2^-9; torch rounds ties to even
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(y, min=2.0 ** -20))), min=-6.0) - 3)
    q = torch.clamp(torch.round(y / step) * step, max=448.0)
    return (torch.copysign(q, blocks) * d).view(rows, -1)[:, :cols]


def exact(case, seed):
    data = {name: t if name == "index" else t.double() for name, t in _inputs(case, seed).items()}
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op in ("norm", "norm8"):
        h = _single(data["x"] + data["residual"]).to(dtype).double()
        r = torch.rsqrt((h * h).sum(1, keepdim=True) / h.shape[1] + EPS)
        w = data["weight"] + case["offset"]
        if op == "norm8":
            return {"sum": h, "y": _exact_values(_single(_single(h * _single(r)) * _single(w)))}
        if not case["train"]:
            return {"sum": h, "y": h * r * w}
        # y_j = w_j h_j r with r = (mean h^2 + eps)^-1/2, so dr/dh_j = -r^3 h_j / k
        dr = (data["dy"] * w * h).sum(1, keepdim=True)
        return {"sum": h, "y": h * r * w, "dx": data["dsum"] + data["dy"] * w * r - dr * r ** 3 * h / h.shape[1],
                "dw": torch.einsum("tk,tk,t->k", data["dy"], h, r[:, 0])}
    if op == "product8":
        x = _exact_values(data["x"])
        if case["form"] == "linear":
            return x @ _exact_values(data["w"]).T
        g, u = x @ _exact_values(data["wg"]).T, x @ _exact_values(data["wu"]).T
        z = g if case["act"] == "silu" else math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
        return g * torch.sigmoid(z) * u
    out = data["y"].clone()
    for i in range(data["a"].shape[0]):
        rows = (data["index"] == i).nonzero()[:, 0]
        out[rows] += data["scale"][i] * ((data["x"][rows] @ data["a"][i].T) @ data["b"][i].T)
    return out
