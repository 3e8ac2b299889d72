"""The 8-bit operators: refusals (no GPU), the quantiser's bits against the 64-bit definition, products against 64-bit
references."""
import pytest
import torch

import ff_reference as ref
import paper_2506_17615_b200 as eq
from paper_2506_17615_b200 import binding
from paper_2506_17615_b200 import feedforward as ff
from test_feedforward import A, ACTS, GB, MANY, SIZES, assert_beside, hard_rows, normal, padded, status_of

gpu = pytest.mark.gpu
CODE = {torch.bfloat16: eq.BF16, torch.float16: eq.FP16, torch.float32: eq.FP32}


# ------------------------------------------------------------------ refusals, sizes (no GPU)

def test_quantize_and_dequantize_refuse_bad_arguments():
    q = dict(x=A, dtype=eq.BF16, rows=4, cols=64, ld=64, codes=A + GB, scales=A + 2 * GB)
    d = dict(codes=A, scales=A + GB, rows=4, cols=64, out=A + 3 * GB, dtype=eq.FP32, ld=64)
    for f, a, free in ((eq.fp8_quantize, q, "x"), (eq.fp8_dequantize, d, "out")):
        for key in ("codes", "scales", free):
            assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
            assert status_of(f, **{**a, key: a[key] + (1 if key == free else 8)}) == binding.ERR_ALIGN
        for bad in (3, -1):
            assert status_of(f, **{**a, "dtype": bad}) == binding.ERR_FORMAT
        for key, bad in (("cols", 0), ("ld", 63), ("rows", GB + 1), ("cols", GB + 1), ("ld", GB + 1)):
            assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
        assert status_of(f, **{**a, "rows": 0, free: 0}) == 0
    assert status_of(eq.fp8_quantize, **{**q, "codes": A + 496}) == binding.ERR_ALIAS          # inside x's last row
    assert status_of(eq.fp8_quantize, **{**q, "scales": A + GB + 240}) == binding.ERR_ALIAS    # inside codes
    assert status_of(eq.fp8_dequantize, **{**d, "out": A + 240}) == binding.ERR_ALIAS


def test_products_refuse_bad_arguments():
    m = dict(a_codes=A, a_scales=A + GB, b_codes=A + 2 * GB, b_scales=A + 3 * GB, m=4, n=8, k=64, out=A + 4 * GB, dtype=eq.FP16, ld=8)
    g = dict(x_codes=A, x_scales=A + GB, g_codes=A + 2 * GB, g_scales=A + 3 * GB, u_codes=A + 5 * GB, u_scales=A + 6 * GB, m=4, f=8,
             k=64, act=0, h=A + 4 * GB, dtype=eq.FP16, ldh=8)
    for f, a, out, n, ld in ((eq.fp8_matmul, m, "out", "n", "ld"), (eq.fp8_gated, g, "h", "f", "ldh")):
        for key in [k for k in a if k.endswith(("codes", "scales"))] + [out]:
            assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
            assert status_of(f, **{**a, key: a[key] + (1 if key == out else 8)}) == binding.ERR_ALIGN
        for key, bad in ((n, 0), ("k", 0), (ld, 7), ("m", GB + 1)):
            assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
        assert status_of(f, **{**a, "dtype": 3}) == binding.ERR_FORMAT
        assert status_of(f, **{**a, out: A + 2 * GB + 16}) == binding.ERR_ALIAS
        assert status_of(f, **{**a, "m": 0, out: 0}) == 0
    assert status_of(eq.fp8_gated, **{**g, "act": 2}) == binding.ERR_FORMAT
    assert status_of(eq.fp8_gated, **{**g, "dtype": eq.FP32}) == binding.ERR_FORMAT            # h has 16 bits
    assert eq.last_cuda_error() == 0


def test_linear_refuses_bad_arguments():
    need = eq.fp8_linear_workspace_bytes(40, 64)
    assert need == 512 + 40 * 64 and eq.fp8_linear_workspace_bytes(1, 64) == 0 and eq.fp8_linear_workspace_bytes(40, 0) == 0
    f = eq.fp8_linear
    a = dict(x=A, dtype=eq.FP16, ldx=64, w_codes=A + GB, w_scales=A + 2 * GB, m=40, n=8, k=64, out=A + 3 * GB, ld=8, workspace=A + 4 * GB,
             workspace_bytes=need)
    for key, off in (("x", 1), ("out", 1), ("w_codes", 8), ("w_scales", 8), ("workspace", 8)):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**a, key: a[key] + off}) == binding.ERR_ALIGN
    for key, bad in (("n", 0), ("k", 0), ("ld", 7), ("ldx", 63), ("m", GB + 1)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
    assert status_of(f, **{**a, "dtype": eq.FP32}) == binding.ERR_FORMAT
    assert status_of(f, **{**a, "workspace_bytes": need - 1}) == binding.ERR_WORKSPACE
    for key, bad in (("out", A + 32), ("out", A + GB + 32), ("workspace", A), ("workspace", A + GB), ("workspace", A + 3 * GB)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_ALIAS
    assert status_of(f, **{**a, "m": 0, "x": 0}) == 0
    assert eq.last_cuda_error() == 0


def test_sizes_of_the_buffers():
    assert eq.fp8_codes_bytes(3, 33) == 3 * 64 and eq.fp8_scales_bytes(1, 1) == 512
    assert eq.fp8_scales_bytes(129, 129) == 2 * 2 * 512
    assert eq.fp8_codes_bytes(4, 0) == 0 and eq.fp8_scales_bytes(0, 64) == 0 and eq.fp8_scales_bytes(4, GB + 1) == 0


def test_what_the_extension_module_refuses():
    cpu = torch.zeros(4, 64, dtype=torch.bfloat16)
    q = ff.Fp8Matrix(torch.zeros(16, dtype=torch.uint8), 4, 64)
    for call in (lambda: ff.fp8_quantize(None), lambda: ff.fp8_quantize(cpu), lambda: ff.fp8_quantize(cpu[0]), lambda: ff.fp8_linear(cpu, q),
                 lambda: ff.fp8_dequantize(q), lambda: ff.fp8_dequantize(q, torch.float64), lambda: ff.fp8_matmul(q, q),
                 lambda: ff.fp8_matmul(q, ff.Fp8Matrix(q.data, 4, 32)), lambda: ff.fp8_gated(q, q, q, dtype=torch.float64),
                 lambda: ff.fp8_gated(q, q, ff.Fp8Matrix(q.data, 5, 64)), lambda: ff._native.matmul8(cpu)):
        with pytest.raises((TypeError, ValueError)):
            call()


# ------------------------------------------------------------------ quantisation

E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1]


def quantize(x):
    """x [rows, cols] float64 -> (code bytes without sign [rows, blocks, 32], scale bytes, what a code is multiplied by), from
    the definition by search"""
    rows, cols = x.shape
    n = -(-cols // 32)
    v = torch.zeros(rows, n * 32, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, n, 32)
    amax = v.abs().amax(-1)
    _, power = torch.frexp(amax)
    e = torch.where(amax > 0, torch.clamp(power - 9, min=-127), torch.full_like(power, -127))
    d = torch.exp2(e.double())
    table = torch.tensor(E4M3, dtype=torch.float64, device=x.device)
    y = (v / d[..., None]).abs()
    hi = torch.searchsorted(table, y.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dlo, dhi = (y - table[lo]).abs(), (table[hi] - y).abs()
    code = torch.where(dlo < dhi, lo, torch.where(dhi < dlo, hi, torch.where(lo % 2 == 0, lo, hi)))
    return code, v < 0, e + 127, d


def values(x):
    code, neg, _, d = quantize(x)
    v = torch.tensor(E4M3, dtype=torch.float64, device=x.device)[code] * torch.where(neg, -1.0, 1.0) * d[..., None]
    return v.reshape(x.shape[0], -1)[:, :x.shape[1]]


def scale_positions(rows, blocks, cols):
    r, b = torch.arange(rows)[:, None], torch.arange(blocks)[None, :]
    return (r // 128 * -(-cols // 128) + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4


def check_matrix(q, x):
    """q holds the codes and scales of x [rows, cols] float64"""
    rows, cols = x.shape
    code, neg, byte, _ = quantize(x)
    flat, signs = code.reshape(rows, -1), neg.reshape(rows, -1)
    assert q.codes.shape == flat.shape
    assert torch.equal((q.codes & 127).long(), flat), "magnitudes differ"
    assert not bool((((q.codes >> 7).bool() != signs) & (flat > 0)).any()), "signs differ"
    pos = scale_positions(rows, byte.shape[1], cols).to(x.device)
    assert torch.equal(q.scales[pos].long(), byte.long()), "scales differ"
    total = -(-cols // 128) * 4
    if total > byte.shape[1]:
        assert not bool(q.scales[scale_positions(rows, total, cols)[:, byte.shape[1]:].to(x.device)].any())


def check_quantized(x):
    q = ff.fp8_quantize(x)
    check_matrix(q, x.double())
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        assert torch.equal(ff.fp8_dequantize(q, dtype).double(), ref.f32(values(x.double())).to(dtype).double()), dtype


@gpu
@pytest.mark.parametrize("dtype", list(CODE))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 16, 0), (3, 17, 0), (5, 31, 2), (128, 256, 0), (129, 257, 7), (33, 500, 12),
                                           (1, 5376, 0), (1300, 96, 0), (300, 2050, 6), (2, 24576, 0), (3, 30001, 0)])
def test_quantize_matches_the_definition(dtype, rows, cols, pad):
    check_quantized(normal(rows, cols, rows + cols, dtype, 3.0, pad))


@gpu
@pytest.mark.parametrize("dtype", list(CODE))
@pytest.mark.parametrize("cols", [32, 64, 333, 512])
def test_quantize_hard_rows(dtype, cols):
    x = hard_rows(cols, dtype)
    ties = torch.tensor([E4M3[i] / 2 + E4M3[i + 1] / 2 for i in range(0, 126, 4)] + [448.0, 460.0, 511.0, -464.0], dtype=torch.float32)
    rows = torch.stack([(ties * s).repeat(-(-cols // len(ties)))[:cols] for s in (1.0, 2.0 ** -7)])
    check_quantized(torch.cat([x, rows.clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype).cuda()]))


@gpu
def test_not_finite_elements_become_nan():
    x = normal(6, 96, 1, torch.bfloat16)
    x[1, 40], x[3, 0], x[4, 95] = float("inf"), float("nan"), float("-inf")
    back = ff.fp8_dequantize(ff.fp8_quantize(x), torch.float32)
    nan = torch.zeros(6, 96, dtype=torch.bool, device="cuda")
    for r, c in ((1, 40), (3, 0), (4, 95)):
        nan[r, c // 32 * 32:(c // 32 + 1) * 32] = True
    assert torch.equal(back.isnan(), nan)
    w = ff.fp8_quantize(normal(40, 96, 2, torch.bfloat16))
    for y in (ff.fp8_linear(x, w), ff.fp8_linear(x.repeat(60, 1), w)[:6]):
        rows = y.isnan()
        assert bool(rows[[1, 3, 4]].all()) and not bool(rows[[0, 2, 5]].any())


@gpu
@pytest.mark.parametrize("dtype", list(CODE))
@pytest.mark.parametrize("cols", [1, 7, 8, 16, 31, 40, 250, 1001, 5002])
def test_rows_that_start_anywhere(cols, dtype):
    """codes, scales and values of rows at every offset are those of aligned rows; nothing is written beside them"""
    rows, wide = 5, (cols + 31) // 32 * 32 + 32
    stream = torch.cuda.current_stream().cuda_stream
    aligned = normal(rows, wide, cols, dtype)[:, :cols]
    want = ff.fp8_quantize(aligned)
    out = torch.empty(rows, wide, device="cuda", dtype=dtype)
    eq.fp8_dequantize(want.codes, want.scales, rows, cols, out, CODE[dtype], wide, stream)
    pos = scale_positions(rows, -(-cols // 32), cols).cuda()
    for offset in (0, 1, 2, 3, 4, 8, 15):
        for ld in (cols, cols + 1, cols + 6, wide):
            store = torch.full((offset + rows * ld + 16,), -77.0, device="cuda", dtype=dtype)
            view = store[offset:].as_strided((rows, cols), (ld, 1))
            view.copy_(aligned)
            got = ff.fp8_quantize(view)
            assert torch.equal(got.codes, want.codes) and torch.equal(got.scales[pos], want.scales[pos])
            store.fill_(-77.0)
            eq.fp8_dequantize(got.codes, got.scales, rows, cols, view, CODE[dtype], ld, stream)
            assert torch.equal(view, out[:, :cols])
            view.fill_(-77.0)
            assert bool((store == -77.0).all())


# ------------------------------------------------------------------ products

@gpu
@pytest.mark.parametrize("m,n,k", SIZES)
def test_products(m, n, k):
    for i, dtype in enumerate((torch.bfloat16, torch.float16)):
        x = normal(m, k, m + n + i, dtype, 1.0, pad=(0, 3, 8)[(m + i) % 3])
        w = normal(n, k, n + k + i, dtype, k ** -0.5)
        wq, xq = ff.fp8_quantize(w), ff.fp8_quantize(x)
        y = ff.fp8_linear(x, wq)
        value, bound = ref.product(values(x.double()), values(w.double()))
        assert y.dtype == dtype
        ref.assert_within(y, value, ref.rounded(value, bound, dtype), "linear")
        assert torch.equal(ff.fp8_matmul(xq, wq, dtype), y)
        y32 = ff.fp8_matmul(xq, wq, torch.float32)
        ref.assert_within(y32, value, ref.rounded(value, bound, torch.float32), "matmul, fp32")
    ff.check()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,k", [(1, 1), (130, 129), (257, 1000), (2688, 128), (1000, 5376), (512, 2697)])
def test_linear_of_few_tokens(n, k, dtype):
    """the same bits as two calls, for rows that start anywhere, and with what is not finite"""
    w = ff.fp8_quantize(normal(n, k, n + k, dtype, k ** -0.5))
    for m in (1, 2, 3, 5, 7, 8, 9, 16, 17):
        for shift in (0, 1, 2, 8):
            store = normal(m, k + shift + 24, m + k, dtype, 1.0)
            x = store[:, shift:shift + k]
            x[m // 2, k // 2] = (float("nan"), float("inf"), -0.0, 60000.0)[(m + shift) % 4]
            got, want = ff.fp8_linear(x, w), ff.fp8_matmul(ff.fp8_quantize(x), w, dtype)
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
    ff.check()


@gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,f,k", SIZES)
def test_gated(act, m, f, k):
    dtype = torch.bfloat16 if (m + f) % 2 else torch.float16
    x = normal(m, k, m + f, dtype, 1.0, pad=(0, 1, 8)[m % 3])
    wg, wu = normal(f, k, f + 1, dtype, 2 * k ** -0.5), normal(f, k, f + 2, dtype, k ** -0.5)
    h = ff.fp8_gated(ff.fp8_quantize(x), ff.fp8_quantize(wg), ff.fp8_quantize(wu), act, dtype)
    value, bound, _, _ = ref.gated(*(values(t.double()) for t in (x, wg, wu)), act)
    ref.assert_within(h, value, ref.rounded(value, bound, dtype), "h")
    ff.check()


@gpu
@pytest.mark.parametrize("m,n,k", MANY)
def test_products_of_many_tiles(m, n, k):
    for dtype in (torch.bfloat16, torch.float32):
        x, w = normal(m, k, 1, torch.bfloat16), normal(n, k, 2, torch.bfloat16, k ** -0.5)
        xq, wq = ff.fp8_quantize(x), ff.fp8_quantize(w)
        y = ff.fp8_matmul(xq, wq, dtype)
        value, bound = ref.product(values(x.double()), values(w.double()))
        ref.assert_within(y, value, ref.rounded(value, bound, dtype), "matmul")
        for first in range(0, m, 1000):
            assert torch.equal(ff.fp8_matmul(ff.fp8_quantize(x[first:first + 1000]), wq, dtype), y[first:first + 1000])
    half = n // 2
    wg, wu = w[:half], w[half:2 * half]
    qg, qu = ff.fp8_quantize(wg), ff.fp8_quantize(wu)
    h = ff.fp8_gated(xq, qg, qu)
    value, bound, _, _ = ref.gated(*(values(t.double()) for t in (x, wg, wu)), eq.ACT_GELU_TANH)
    ref.assert_within(h, value, ref.rounded(value, bound, torch.bfloat16), "h")
    ff.check()


@gpu
@pytest.mark.parametrize("parts", [1, 2, 5, 8])
def test_every_scale_of_a_stage_is_used(parts):
    """elements alone in their blocks, of very different sizes: a block's power of two that were another's would show"""
    k = 128 * parts
    for m in (1, 200):
        x, w = torch.zeros(m, k, device="cuda"), torch.zeros(60, k, device="cuda")
        for b in range(k // 32):
            x[:, b * 32 + b % 32] = 2.0 ** (b % 9) * torch.arange(1, m + 1, device="cuda").remainder(7).add(1)
            w[:, b * 32 + b % 32] = 2.0 ** -(b % 9) * (1 + torch.arange(60, device="cuda") % 5)
        x, w = x.bfloat16(), w.bfloat16()
        want = x.double() @ w.double().T                            # integers: every sum is exact
        assert torch.equal(ff.fp8_matmul(ff.fp8_quantize(x), ff.fp8_quantize(w), torch.float32).double(), want)
    ff.check()


@gpu
def test_no_tokens_streams_and_graphs():
    x, w = normal(300, 200, 1, torch.bfloat16), ff.fp8_quantize(normal(256, 200, 2, torch.bfloat16, 0.1))
    none = ff.fp8_quantize(x[:0])
    assert ff.fp8_matmul(none, w).shape == (0, 256) and ff.fp8_gated(none, w, w).shape == (0, 256)
    assert ff.fp8_dequantize(none).shape == (0, 200) and ff.fp8_linear(x[:0], w).shape == (0, 256)

    def everything():
        q = ff.fp8_quantize(x)
        return ff.fp8_linear(x, w), ff.fp8_linear(x[:3], w), ff.fp8_gated(q, w, w), ff.fp8_dequantize(q)

    want = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for got in [everything() for _ in range(3)]:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    asking = x.clone().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        ff.fp8_linear(asking, w)
    with pytest.raises(ValueError):
        ff.fp8_linear(x.float(), w)
    with torch.no_grad():
        assert torch.equal(ff.fp8_linear(asking, w), want[0])


@gpu
def test_launch_errors_come_back(monkeypatch):
    x = normal(4, 64, 1, torch.bfloat16)
    q = ff.fp8_quantize(x)
    monkeypatch.setenv("EQUARX_INJECT_LAUNCH_ERROR", "719")
    for call in (lambda: ff.fp8_quantize(x), lambda: ff.fp8_linear(x, q), lambda: ff.fp8_gated(q, q, q), lambda: ff.fp8_dequantize(q)):
        with pytest.raises(eq.EquarxError) as err:
            call()
        assert err.value.status == binding.ERR_CUDA and eq.last_cuda_error() == 719
    monkeypatch.delenv("EQUARX_INJECT_LAUNCH_ERROR")
    ff.fp8_linear(x, q)
    ff.check()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("beside", [0, 8])
@pytest.mark.parametrize("m,n,k", [(3, 33, 75), (300, 130, 101), (261, 5, 67), (1500, 541, 259), (2100, 1663, 126)])
def test_what_lies_beside_an_output_stays(dtype, beside, m, n, k):
    """through the C ABI: the bits of dense outputs, and nothing past an output's last column, whose row goes on to a multiple of 16 bytes"""
    stream = torch.cuda.current_stream().cuda_stream
    x, w = normal(m, k, 1, dtype), ff.fp8_quantize(normal(n, k, 2, dtype, 0.1))
    q = ff.fp8_quantize(x)
    nb = eq.fp8_linear_workspace_bytes(m, k)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    for call, want in (
            (lambda v, ld: eq.fp8_matmul(q.codes, q.scales, w.codes, w.scales, m, n, k, v, CODE[dtype], ld, stream), ff.fp8_matmul(q, w, dtype)),
            (lambda v, ld: eq.fp8_linear(x, CODE[dtype], k, w.codes, w.scales, m, n, k, v, ld, ws, nb, stream), ff.fp8_linear(x, w)),
            (lambda v, ld: eq.fp8_gated(q.codes, q.scales, w.codes, w.scales, w.codes, w.scales, m, n, k, eq.ACT_SILU, v, CODE[dtype], ld, stream),
             ff.fp8_gated(q, w, w, eq.ACT_SILU, dtype))):
        store, ld, view = padded(m, n, dtype, beside)
        call(view, ld)
        assert torch.equal(view, want)
        assert_beside(store, n)
    ff.check()
