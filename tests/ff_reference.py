"""Plain 64-bit references of the feed-forward operators, and bounds on what 16-bit outputs may be off.

Bounds.  A product of K terms summed in fp32 in any order is off by at most K * 2^-23 * sum |a b| (the
tensor cores may truncate where a CPU would round, hence 2^-23 and not 2^-24).  Rounding to a 16-bit type
adds 2^-8 (bf16) or 2^-11 (fp16) of the value, and 2^-25 where fp16 has run out of exponent.  The
activation is evaluated in fp32 with two hardware approximations of a few units in the last place each:
2^-19 of its value covers them, and an error e of its argument moves it by at most 1.2 e (the largest
slopes of silu and gelu are 1.10 and 1.13).
"""
import math

import torch

import paper_2506_17615_b200 as eq

E2M1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
ACC = 2.0 ** -23
ACT_ERR = 2.0 ** -19


def f32(t):
    return t.to(torch.float32).to(torch.float64)


def nearest_code(y):
    """magnitude index of E2M1: nearest, ties to the even index, 6 and above saturate (64-bit, by search)"""
    a = y.abs().unsqueeze(-1)
    dist = (a - E2M1.to(y.device)).abs()
    best = dist.amin(-1, keepdim=True)
    hit = dist == best
    idx = torch.arange(8, device=y.device)
    cand = torch.where(hit, idx, torch.full_like(idx, 99))
    first = cand.amin(-1)
    last = torch.where(hit, idx, torch.full_like(idx, -1)).amax(-1)
    return torch.where(first % 2 == 0, first, last)


def e4m3_nearest(y):
    """nearest non-negative E4M3 value and its byte, ties to the even byte (64-bit, by search)"""
    byte = torch.arange(0, 127, device=y.device)
    e, m = byte // 8, byte % 8
    val = torch.where(e == 0, m.double() * 2.0 ** -9, (1 + m.double() / 8) * torch.exp2(e.double() - 7))
    hi = torch.searchsorted(val, y.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dlo, dhi = (y - val[lo]).abs(), (val[hi] - y).abs()
    pick = torch.where(dlo < dhi, lo, torch.where(dhi < dlo, hi, torch.where(lo % 2 == 0, lo, hi)))
    return val[pick], pick


def quantize(x, fmt):
    """x [rows, cols] float64 -> (signed magnitude indexes [rows, blocks, size], sign of every element,
    scale bytes [rows, blocks], what a code is multiplied by [rows, blocks], row factors [rows])"""
    rows, cols = x.shape
    size = 32 if fmt == eq.FP4_MX else 16
    n = -(-cols // size)
    v = torch.zeros(rows, n * size, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, n, size)
    amax = v.abs().amax(-1)
    if fmt == eq.FP4_MX:
        frac, power = torch.frexp(amax)
        e = torch.where(amax > 0, torch.clamp(power - 3, min=-127), torch.full_like(power, -127))
        d = torch.exp2(e.double())
        return nearest_code(v / d[..., None]), v < 0, e + 127, d, None
    top = amax.amax(1, keepdim=True)
    live = top >= 2.0 ** -100
    safe = torch.where(live, top, torch.ones_like(top))
    g = torch.where(live, f32(safe / 2688), torch.zeros_like(safe))
    s, byte = e4m3_nearest(torch.clamp(f32(amax * torch.where(live, f32(448 / safe), torch.zeros_like(safe))), max=448.0))
    d = f32(s * g)
    ok = s > 0
    y = torch.where(ok[..., None], f32(v * f32(1 / torch.where(ok, d, torch.ones_like(d)))[..., None]), torch.zeros_like(v))
    return nearest_code(y), v < 0, byte, d, g[:, 0]


def values(x, fmt):
    code, neg, _, d, _ = quantize(x, fmt)
    v = E2M1.to(x.device)[code] * torch.where(neg, -1.0, 1.0) * d[..., None]
    return v.reshape(x.shape[0], -1)[:, :x.shape[1]]


def scale_positions(rows, blocks, cols, fmt):
    """byte position of every (row, block) in the tiled scale buffer, from the layout's definition"""
    tiles = -(-cols // 256) * (2 if fmt == eq.FP4_MX else 4)
    r = torch.arange(rows)[:, None]
    b = torch.arange(blocks)[None, :]
    return (r // 128 * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4


def act(g, kind):
    if kind == eq.ACT_SILU:
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def slope(g, kind):
    if kind == eq.ACT_SILU:
        s = torch.sigmoid(g)
        return s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def product(a, b):
    """a b^T and the bound on an fp32 sum of it"""
    return a @ b.T, a.shape[1] * ACC * (a.abs() @ b.abs().T)


def rounded(value, bound, dtype):
    return bound + UNIT[dtype] * (value.abs() + bound) + TINY[dtype]


def gated(x, wg, wu, kind):
    """h and the bound on it before rounding, with g, u and their bounds"""
    (g, eg), (u, eu) = product(x, wg), product(x, wu)
    a = act(g, kind)
    ea = 1.2 * eg + ACT_ERR * a.abs() + 2.0 ** -126
    return a * u, ea * u.abs() + a.abs() * eu + ea * eu + 2.0 ** -23 * (a * u).abs(), (g, eg), (u, eu)


def assert_within(got, value, bound, what):
    got = got.double()
    assert got.shape == value.shape, what
    bad = ~((got - value).abs() <= bound)
    assert not bool(bad.any()), \
        f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, worst ratio " \
        f"{float(((got - value).abs() / bound).nan_to_num(float('inf')).max()):.3g}, first at {bad.nonzero()[0].tolist()}"
