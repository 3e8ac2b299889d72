"""The residual addition with RMS norm: refusals (no GPU), and the kernels against 64-bit references.

The forward pass is defined step by step in fp32, with a row's sum of squares in fp64, so its results are compared bit for
bit with the definition in torch.  (A row's factor r could differ where its exact value lies within 2^-45 of the border between two
fp32 numbers: one row in 2^20.)

Bounds of the gradients, relative to the sums of magnitudes: n, g and their product take 4 roundings to fp32; a row's sum
passes 4 pairs of columns for each 1792 columns of the row, and 11 steps of a tree.  A sum over rows passes fewer
additions than there are rows, and 10 more.
"""
import pytest
import torch

import ff_reference as ref
import paper_2506_17615_b200 as eq
from paper_2506_17615_b200 import binding
from paper_2506_17615_b200 import feedforward as ff
from paper_2506_17615_b200 import norm
from test_feedforward import A, GB, leaves, normal, status_of
from test_fp8 import check_matrix

gpu = pytest.mark.gpu
EPS = 2.0 ** -24
CODE = {torch.bfloat16: eq.BF16, torch.float16: eq.FP16, torch.float32: eq.FP32}
TYPES = [torch.bfloat16, torch.float16]


# ------------------------------------------------------------------ refusals (no GPU)

def forward_args():
    return dict(x=A, ldx=64, residual=A + GB, ldr=64, weight=A + 2 * GB, dtype=eq.BF16, weight_dtype=eq.FP32, rows=4, cols=64, eps=1e-6,
                offset=0.0, sum=A + 3 * GB, lds=64)


def test_forward_refuses_bad_arguments():
    plain = dict(forward_args(), y=A + 4 * GB, ldy=64, factors=A + 5 * GB)
    eight = dict(forward_args(), codes=A + 4 * GB, scales=A + 5 * GB)
    for f, a in ((eq.add_rms_norm, plain), (eq.add_rms_norm_fp8, eight)):
        pointers = [k for k in a if isinstance(a[k], int) and a[k] >= A]
        for key in pointers:
            if key != "factors":
                assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL, key
            assert status_of(f, **{**a, key: a[key] + 1}) == binding.ERR_ALIGN, key
        for key, bad in (("dtype", eq.FP32), ("dtype", -1), ("weight_dtype", eq.FP16), ("weight_dtype", 3)):
            assert status_of(f, **{**a, key: bad}) == binding.ERR_FORMAT
        for key, bad in (("cols", 0), ("cols", GB + 1), ("rows", GB + 1), ("ldx", 63), ("ldr", 63), ("lds", 63)):
            assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
        for key, bad in (("eps", -1e-9), ("eps", float("nan")), ("eps", float("inf")), ("offset", float("nan")), ("offset", float("inf"))):
            assert status_of(f, **{**a, key: bad}) == binding.ERR_VALUE
        assert status_of(f, **{**a, "rows": 0, "x": 0}) == 0
        # the sum may be an input, but not a shifted one, one of another stride, the weight or another output
        for bad in (A + 2, A + GB + 64, A + 2 * GB, A + 4 * GB):
            assert status_of(f, **{**a, "sum": bad}) == binding.ERR_ALIAS
        assert status_of(f, **{**a, "sum": A, "lds": 72}) == binding.ERR_ALIAS
        assert status_of(f, **{**a, pointers[-2]: A}) == binding.ERR_ALIAS
    assert status_of(eq.add_rms_norm, **{**plain, "ldy": 63}) == binding.ERR_COUNT
    assert status_of(eq.add_rms_norm, **{**plain, "factors": A + 3 * GB + 4}) == binding.ERR_ALIAS
    assert eq.last_cuda_error() == 0


def test_backward_refuses_bad_arguments():
    need = eq.add_rms_norm_backward_workspace_bytes(40, 64)
    assert need == 20 * 64 * 4 and eq.add_rms_norm_backward_workspace_bytes(40, 0) == 0
    assert eq.add_rms_norm_backward_workspace_bytes(4, 64) == 0                  # a few rows need none
    a = dict(dy=A, lddy=64, dsum=A + GB, ldds=64, sum=A + 2 * GB, lds=64, factors=A + 3 * GB, weight=A + 4 * GB, dtype=eq.FP16,
             weight_dtype=eq.FP16, rows=40, cols=64, offset=1.0, dx=A + 5 * GB, lddx=64, dweight=A + 6 * GB, workspace=A + 7 * GB,
             workspace_bytes=need)
    f = eq.add_rms_norm_backward
    for key in ("dy", "sum", "factors", "weight", "dx", "workspace"):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
    for key in ("dy", "dsum", "sum", "factors", "weight", "dx", "dweight", "workspace"):
        assert status_of(f, **{**a, key: a[key] + 1}) == binding.ERR_ALIGN
    for key, bad in (("dtype", eq.FP32), ("weight_dtype", eq.BF16)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_FORMAT
    for key, bad in (("cols", 0), ("lddy", 63), ("ldds", 63), ("lds", 63), ("lddx", 63), ("rows", GB + 1)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
    assert status_of(f, **{**a, "offset": float("nan")}) == binding.ERR_VALUE
    assert status_of(f, **{**a, "workspace_bytes": need - 1}) == binding.ERR_WORKSPACE
    for key, bad in (("dx", A), ("dx", A + GB), ("dweight", A + 4 * GB), ("dweight", A + 5 * GB), ("workspace", A + 2 * GB)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_ALIAS
    assert eq.last_cuda_error() == 0


def test_what_the_extension_module_refuses():
    cpu, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.bfloat16)
    for call in (lambda: norm.add_rms_norm(cpu, None, w), lambda: norm.add_rms_norm(None, None, w), lambda: norm.add_rms_norm(cpu[0], None, w),
                 lambda: norm.add_rms_norm_fp8(cpu, cpu, w), lambda: norm.add_rms_norm_backward(cpu, None, cpu, w, w),
                 lambda: norm._native.add_rms_norm(cpu)):
        with pytest.raises((TypeError, ValueError)):
            call()
    assert "VALUE" in eq.status_string(binding.ERR_VALUE)


# ------------------------------------------------------------------ forward

def inputs(rows, cols, seed, dtype, wtype, offset, pad=0):
    x, residual = normal(rows, cols, seed, dtype, 1.0, pad), normal(rows, cols, seed + 1, dtype, 3.0, pad)
    x[:, cols // 2] *= 40.0
    w = (normal(1, cols, seed + 2, torch.float32, 0.3)[0] + (1.0 - offset)).to(wtype)
    return x, residual, w


def definition(x, residual, w, eps, offset):
    """sum, r and the normalised rows, step by step"""
    total = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h = total.float()
    r = (1.0 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)).float()
    return total, r, (h * r) * (w.float() + offset)


SHAPES = [(1, 1, 0), (1, 8, 0), (3, 17, 0), (5, 31, 2), (2, 512, 0), (129, 257, 7), (33, 500, 12), (1, 3840, 0), (64, 5376, 0), (777, 1250, 46),
          (300, 2050, 6), (2000, 96, 0), (3, 2056, 0), (400, 4100, 4), (2, 7168, 0), (2, 8192, 0), (3, 8960, 0), (3, 8968, 0), (2, 20001, 0), (1, 40000, 16)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", SHAPES)
def test_forward_matches_the_definition(dtype, rows, cols, pad):
    for wtype, offset in ((dtype, 0.0), (torch.float32, 1.0)):
        x, residual, w = inputs(rows, cols, rows + cols, dtype, wtype, offset, pad)
        for res in (residual, None):
            total, r, v = definition(x, res, w, 1e-6, offset)
            y, s, factors = norm.add_rms_norm(x, res, w, 1e-6, offset, save=True)
            assert torch.equal(s, total) and (res is not None or s is x)
            assert torch.equal(factors, r[:, 0]) and torch.equal(y, v.to(dtype))
            assert torch.equal(norm.add_rms_norm(x, res, w, 1e-6, offset)[0], y)
            q, s = norm.add_rms_norm_fp8(x, res, w, 1e-6, offset)
            assert torch.equal(s, total)
            check_matrix(q, v.double())
            # against the formula in 64 bits: four roundings before the last
            h = total.double()
            exact = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * (w.double() + offset)
            ref.assert_within(y, exact, ref.rounded(exact, 4 * EPS * (h * r.double()).abs() * (w.double().abs() + offset), dtype), "y")


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 16, 40, 250, 1001])
def test_rows_that_start_anywhere(cols, dtype):
    """inputs, weight and outputs at every offset give the bits of aligned ones, and nothing is written beside them; the sum in
    place of the residual, too"""
    rows, stream = 5, torch.cuda.current_stream().cuda_stream
    x, residual, w = inputs(rows, cols, 3, dtype, dtype, 1.0)
    y, s, factors = norm.add_rms_norm(x, residual, w, 1e-6, 1.0, save=True)
    q, _ = norm.add_rms_norm_fp8(x, residual, w, 1e-6, 1.0)
    for offset in (0, 1, 2, 4, 8):
        for ld in (cols, cols + 1, cols + 6, (cols + 15) // 16 * 16 + 16):
            def place(t):
                store = torch.full((offset + rows * ld + 16,), -77.0, device="cuda", dtype=dtype)
                view = store[offset:].as_strided((rows, cols), (ld, 1))
                return store, view.copy_(t) if t is not None else view

            (_, vx), (sr, vr), (ss, vs), (sy, vy) = place(x), place(residual), place(None), place(None)
            vw = torch.empty(cols + offset, device="cuda", dtype=dtype)[offset:].copy_(w)
            code = CODE[dtype]
            f = torch.empty(rows, device="cuda")
            eq.add_rms_norm(vx, ld, vr, ld, vw, code, code, rows, cols, 1e-6, 1.0, vs, ld, vy, ld, f, stream)
            assert torch.equal(vs, s) and torch.equal(vy, y) and torch.equal(f, factors)
            for store, view in ((ss, vs), (sy, vy)):
                view.fill_(-77.0)
                assert bool((store == -77.0).all())
            got = ff.Fp8Matrix(torch.zeros_like(q.data), rows, cols)
            eq.add_rms_norm_fp8(vx, ld, vr, ld, vw, code, code, rows, cols, 1e-6, 1.0, vr, ld, got.codes, got.scales, stream)
            assert torch.equal(vr, s) and torch.equal(ff.fp8_dequantize(got, torch.float32), ff.fp8_dequantize(q, torch.float32))
            vr.fill_(-77.0)
            assert bool((sr == -77.0).all())
            eq.add_rms_norm(vx, ld, vs.copy_(residual), ld, vw, code, code, rows, cols, 1e-6, 1.0, vx, ld, vy, ld, 0, stream)
            assert torch.equal(vx, s) and torch.equal(vy, y)


@gpu
@pytest.mark.parametrize("cols", [40, 16400])
def test_rows_of_zeros_and_not_finite_ones(cols):
    dtype = torch.bfloat16
    x, residual, w = inputs(6, cols, 1, dtype, dtype, 0.0)
    x[1], residual[1] = 0.0, 0.0
    x[2, 3], x[3, 0], residual[4, cols - 1] = float("inf"), float("nan"), float("-inf")
    y, s = norm.add_rms_norm(x, residual, w)
    q, _ = norm.add_rms_norm_fp8(x, residual, w)
    back = ff.fp8_dequantize(q, torch.float32)
    clean = [0, 5]
    assert torch.equal(y[clean], norm.add_rms_norm(x[clean], residual[clean], w)[0])
    assert not bool(y[1].any()) and not bool(back[1].any())                     # zeros, with eps
    # r is 0 beside an infinite element: it becomes NaN, the others 0; beside NaN all are NaN
    for row, col in ((2, 3), (4, cols - 1)):
        assert bool(y[row, col].isnan()) and int(y[row].isnan().sum()) == 1 and not bool(y[row].nan_to_num(0.0).any())
        block = col // 32 * 32
        assert bool(back[row, block:block + 32].isnan().all()) and not bool(back[row, :block].any())
    assert bool(y[3].isnan().all()) and bool(back[3].isnan().all())
    # without eps, zeros have no norm; codes past the last column are 0 all the same
    y, _ = norm.add_rms_norm(x, residual, w, 0.0)
    q, _ = norm.add_rms_norm_fp8(x, residual, w, 0.0)
    assert bool(y[1].isnan().all()) and torch.equal(y[clean], norm.add_rms_norm(x[clean], residual[clean], w, 0.0)[0])
    assert not bool(q.codes[:, cols:].any())


@gpu
def test_large_and_small_rows():
    """squares beyond fp32's range on both sides"""
    w = torch.ones(100, dtype=torch.bfloat16, device="cuda")
    base = normal(4, 100, 1, torch.bfloat16)
    want = definition(base, None, w, 0.0, 0.0)[2]
    for scale in (2.0 ** 100, 2.0 ** -100):
        x = base * scale
        y, _, r = norm.add_rms_norm(x, None, w, 0.0, save=True)
        assert torch.equal(y, want.to(torch.bfloat16))
        dx, dw = norm.add_rms_norm_backward(base, None, x, r, w)
        assert bool(dx.isfinite().all()) and bool(dw.isfinite().all()) and bool(dw.any())


# ------------------------------------------------------------------ gradients

def gradients(dy, dsum, total, w, eps, offset):
    """(dx, bound), (dw, bound) in 64 bits"""
    h, dy, w = total.double(), dy.double(), w.double() + offset
    rows, cols = h.shape
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + eps)
    n, g = h * r, dy * w
    ds = torch.zeros_like(h) if dsum is None else dsum.double()
    dx = ds + r * (g - n * (g * n).mean(1, keepdim=True))
    steps = 4 * -(-cols // 1792) + 11 + 4
    ec = steps * EPS * (g * n).abs().mean(1, keepdim=True)
    # dx = dsum + r g - c n takes two more roundings, of dsum + r g (no more than |dx| + |c n|) and of dx
    ex = r * (6 * EPS * (g.abs() + (n * (g * n).mean(1, keepdim=True)).abs()) + n.abs() * ec) + 2 * EPS * dx.abs()
    return (dx, ex), ((dy * n).sum(0), (rows + 10 + 4) * EPS * (dy * n).abs().sum(0))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", SHAPES + [(2, 842, 0), (16, 5376, 0), (17, 1001, 3), (16, 8960, 0), (33, 40, 0), (7, 20001, 0), (1000, 64, 0), (5000, 40, 0), (450, 16400, 0), (450, 17001, 0)])
def test_gradients(dtype, rows, cols, pad):
    for wtype, offset in ((dtype, 1.0), (torch.float32, 0.0)):
        x, residual, w = inputs(rows, cols, rows + cols, dtype, wtype, offset, pad)
        dy, dsum = normal(rows, cols, 7, dtype, 1.0, pad), normal(rows, cols, 8, dtype)
        _, s, factors = norm.add_rms_norm(x, residual, w, 1e-6, offset, save=True)
        for extra in (dsum, None):
            got = norm.add_rms_norm_backward(dy, extra, s, factors, w, offset)
            (dx, ex), (dw, ew) = gradients(dy, extra, s, w, 1e-6, offset)
            assert got[0].dtype == dtype and got[1].dtype == wtype
            ref.assert_within(got[0], dx, ref.rounded(dx, ex, dtype), "dx")
            ref.assert_within(got[1], dw, ref.rounded(dw, ew, wtype), "dw")
            again = norm.add_rms_norm_backward(dy, extra, s, factors, w, offset)
            assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]), "not deterministic"


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,shift", [(9001, 256, 0), (2999, 40, 1), (7000, 33, 0), (1777, 848, 0), (1301, 1792, 0), (1201, 1250, 2), (1999, 2048, 0),
                                             (1500, 2048, 1), (1333, 3584, 0), (1000, 3581, 0), (1200, 5374, 0), (1000, 5375, 0), (600, 8191, 0),
                                             (600, 8192, 2), (300, 8200, 0)])
def test_gradients_of_many_rows(dtype, rows, cols, shift):
    """several rows at a time in a CTA, and rows that are read by pairs or elements, within their memory; dx does not ask for dweight"""
    code, stream = eq.BF16 if dtype == torch.bfloat16 else eq.FP16, torch.cuda.current_stream().cuda_stream
    x, residual, w = inputs(rows, cols, rows + cols, dtype, dtype, 0.0)
    dy, dsum = normal(rows, cols + 8, 7, dtype)[:, shift:shift + cols], normal(rows, cols, 8, dtype)
    _, s, factors = norm.add_rms_norm(x, residual, w, save=True)
    nb = eq.add_rms_norm_backward_workspace_bytes(rows, cols)
    store, ws = torch.full((rows * cols + 16,), -77.0, device="cuda", dtype=dtype), torch.full((nb + 512,), 77, device="cuda", dtype=torch.uint8)
    dx, dw = store[8:8 + rows * cols].view(rows, cols), torch.full((cols + 16,), -77.0, device="cuda", dtype=dtype)
    for extra in (dsum, None):
        eq.add_rms_norm_backward(dy, cols + 8, extra, cols, s, cols, factors, w, code, code, rows, cols, 0.0, dx, cols, dw[8:], ws[256:], nb,
                                 stream)
        (vx, ex), (vw, ew) = gradients(dy, extra, s, w, 1e-6, 0.0)
        ref.assert_within(dx, vx, ref.rounded(vx, ex, dtype), "dx")
        ref.assert_within(dw[8:8 + cols], vw, ref.rounded(vw, ew, dtype), "dw")
        bits = dx.clone()
        eq.add_rms_norm_backward(dy, cols + 8, extra, cols, s, cols, factors, w, code, code, rows, cols, 0.0, dx, cols, 0, 0, 0, stream)
        assert torch.equal(dx, bits)
    for t, n, fill in ((store, 8, -77.0), (dw, 8, -77.0), (ws, 256, 77)):
        assert bool((t[:n] == fill).all()) and bool((t[-n:] == fill).all())


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1185, 3840, 0), (8192, 3840, 0), (1200, 3585, 0), (1700, 3592, 8), (2000, 3714, 2), (1500, 3839, 1),
                                           (1185, 3841, 0), (1185, 3584, 0), (1185, 2688, 0), (1185, 2689, 0), (1184, 3840, 0), (888, 3840, 0), (889, 3840, 0)])
def test_gradients_of_long_batches(dtype, rows, cols, pad):
    """sizes at whose borders the form of the launch changes: how many groups an SM has, and whether one CTA has them all"""
    x, residual, w = inputs(rows, cols, rows + cols, dtype, dtype, 1.0, pad)
    dy, dsum = normal(rows, cols, 7, dtype, 1.0, pad), normal(rows, cols, 8, dtype)
    _, s, factors = norm.add_rms_norm(x, residual, w, 1e-6, 1.0, save=True)
    got = norm.add_rms_norm_backward(dy, dsum, s, factors, w, 1.0)
    (dx, ex), (dw, ew) = gradients(dy, dsum, s, w, 1e-6, 1.0)
    ref.assert_within(got[0], dx, ref.rounded(dx, ex, dtype), "dx")
    ref.assert_within(got[1], dw, ref.rounded(dw, ew, dtype), "dw")
    again = norm.add_rms_norm_backward(dy, dsum, s, factors, w, 1.0)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]), "not deterministic"


@gpu
@pytest.mark.parametrize("rows,cols", [(4, 40), (60, 300)])
def test_gradients_against_differences(rows, cols):
    """<gradient, v> against a central difference of the 64-bit formula along v; the difference's own error is O(step^2)"""
    dtype, offset = torch.float16, 1.0
    x, residual, w = inputs(rows, cols, 5, dtype, torch.float32, offset)
    dy, dsum = normal(rows, cols, 7, dtype), normal(rows, cols, 8, dtype)
    _, s, factors = norm.add_rms_norm(x, residual, w, 1e-6, offset, save=True)
    got = norm.add_rms_norm_backward(dy, dsum, s, factors, w, offset)
    bounds = gradients(dy, dsum, s, w, 1e-6, offset)

    def loss(h, w):
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * (w + offset)
        return (dy.double() * y).sum() + (dsum.double() * h).sum()

    args = [s.double(), w.double()]
    for i, (g, (v, e)) in enumerate(zip(got, bounds)):
        gen = torch.Generator().manual_seed(10 + i)
        direction = torch.randn(g.shape, generator=gen, dtype=torch.float64).cuda()
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + 1e-4 * direction, args[i] - 1e-4 * direction
        numeric = (loss(*plus) - loss(*minus)) / 2e-4
        tol = (ref.rounded(v, e, g.dtype) * direction.abs()).sum() + 1e-5 * numeric.abs() + 1e-6
        assert abs(float((g.double() * direction).sum() - numeric)) <= float(tol), i


@gpu
@pytest.mark.parametrize("offset", [1, 2, 8])
@pytest.mark.parametrize("rows,cols", [(5, 40), (200, 264), (3, 16400)])
def test_backward_of_views_that_start_anywhere(rows, cols, offset):
    dtype, stream = torch.bfloat16, torch.cuda.current_stream().cuda_stream
    x, residual, w = inputs(rows, cols, 5, dtype, dtype, 0.0)
    dy, dsum = normal(rows, cols, 7, dtype), normal(rows, cols, 8, dtype)
    _, s, factors = norm.add_rms_norm(x, residual, w, save=True)
    want = gradients(dy, dsum, s, w, 1e-6, 0.0)
    ld = cols + 3
    stores = [torch.full((offset + rows * ld + 16,), -77.0, device="cuda", dtype=dtype) for _ in range(4)]
    vy, vd, vs, vx = (t[offset:].as_strided((rows, cols), (ld, 1)) for t in stores)
    vy.copy_(dy), vd.copy_(dsum), vs.copy_(s)
    dw = torch.full((cols + offset + 8,), -77.0, device="cuda", dtype=dtype)
    nb = eq.add_rms_norm_backward_workspace_bytes(rows, cols)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    eq.add_rms_norm_backward(vy, ld, vd, ld, vs, ld, factors, w, eq.BF16, eq.BF16, rows, cols, 0.0, vx, ld, dw[offset:], ws, nb, stream)
    ref.assert_within(vx, want[0][0], ref.rounded(*want[0], dtype), "dx")
    ref.assert_within(dw[offset:offset + cols], want[1][0], ref.rounded(*want[1], dtype), "dw")
    vx.fill_(-77.0)
    assert bool((stores[3] == -77.0).all()) and bool((dw[:offset] == -77.0).all()) and bool((dw[offset + cols:] == -77.0).all())
    # no gradient of the weight: no workspace
    eq.add_rms_norm_backward(vy, ld, vd, ld, vs, ld, factors, w, eq.BF16, eq.BF16, rows, cols, 0.0, vx, ld, 0, 0, 0, stream)
    ref.assert_within(vx, want[0][0], ref.rounded(*want[0], dtype), "dx")


@gpu
@pytest.mark.parametrize("rows", [5, 600])
def test_autograd(rows):
    dtype, cols = torch.bfloat16, 72
    x, residual, w = inputs(rows, cols, 1, dtype, torch.float32, 0.0)
    dy, ds = normal(rows, cols, 4, dtype), normal(rows, cols, 5, dtype)
    y, s, factors = norm.add_rms_norm(x, residual, w, save=True)
    dx, dw = norm.add_rms_norm_backward(dy, ds, s, factors, w)
    args = leaves(x, residual, w)
    out = norm.add_rms_norm(*args, save=True)
    assert all(torch.equal(a, b) for a, b in zip(out, (y, s, factors))) and not out[2].requires_grad
    torch.autograd.backward([out[0], out[1]], [dy, ds])
    assert torch.equal(args[0].grad, dx) and torch.equal(args[1].grad, dx) and torch.equal(args[2].grad, dw)
    args[0].grad.zero_()                                           # the two are not one tensor
    assert torch.equal(args[1].grad, dx)
    # only y, only the sum, expanded and transposed gradients, no residual
    args = leaves(x, residual, w)
    norm.add_rms_norm(*args)[0].backward(dy)
    assert torch.equal(args[0].grad, norm.add_rms_norm_backward(dy, None, s, factors, w)[0])
    args = leaves(x, residual, w)
    norm.add_rms_norm(*args)[1].backward(ds)
    assert torch.equal(args[0].grad, ds) and torch.equal(args[1].grad, ds) and args[2].grad is None
    for grad in (torch.ones(1, 1, dtype=dtype, device="cuda").expand(rows, cols), dy.T.contiguous().T):
        args = leaves(x, residual, w)
        norm.add_rms_norm(*args)[0].backward(grad)
        assert torch.equal(args[2].grad, norm.add_rms_norm_backward(grad.contiguous(), None, s, factors, w)[1])
    leaf, weight = leaves(x, w)
    y0, same = norm.add_rms_norm(leaf, None, weight)
    assert same is leaf
    (y0 * 2).backward(dy)
    _, _, f0 = norm.add_rms_norm(x, None, w, save=True)
    assert torch.equal(leaf.grad, norm.add_rms_norm_backward(dy * 2, None, x, f0, w)[0])
    with pytest.raises(ValueError, match="no_grad"):
        norm.add_rms_norm_fp8(leaf, None, w)
    with torch.no_grad():
        assert not norm.add_rms_norm(leaf, None, weight)[0].requires_grad
        norm.add_rms_norm_fp8(leaf, None, weight)
    grad, = torch.autograd.grad(norm.add_rms_norm(leaf, None, w)[0].float().square().sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.float().sum().backward()
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="tangent"):
            norm.add_rms_norm(torch.autograd.forward_ad.make_dual(x, x), None, w)


@gpu
def test_no_rows_streams_graphs_far_strides():
    dtype = torch.bfloat16
    x, residual, w = inputs(70, 96, 1, dtype, dtype, 0.0)
    y, s = norm.add_rms_norm(x[:0], residual[:0], w)
    assert y.shape == s.shape == (0, 96) and norm.add_rms_norm_fp8(x[:0], residual[:0], w)[0].rows == 0
    dx, dw = norm.add_rms_norm_backward(y, None, s, torch.empty(0, device="cuda"), w)
    assert dx.shape == (0, 96) and not bool(dw.any())

    def everything(x=x, residual=residual):
        y, s, f = norm.add_rms_norm(x, residual, w, save=True)
        q, _ = norm.add_rms_norm_fp8(x, residual, w)
        return (y, s, f, ff.fp8_dequantize(q), *norm.add_rms_norm_backward(y, s, s, f, w))

    want = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for got in [everything() for _ in range(3)]:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                                             # two graphs share a pool of memory
        graphs.append((torch.cuda.CUDAGraph(), None))
        with torch.cuda.graph(graphs[-1][0]):
            got = everything()
        graphs[-1] = (graphs[-1][0], got)
    for graph, got in graphs * 2:
        for t in got:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # rows 2^26 elements apart: the last ones lie more than 2^32 elements after the first
    ld = 1 << 26
    store = torch.empty(69 * ld + 4096, dtype=dtype, device="cuda")
    fx, fr = store.as_strided((70, 96), (ld, 1)), store.as_strided((70, 96), (ld, 1), 1024)
    fx.copy_(x), fr.copy_(residual)
    for a, b in zip(everything(fx, fr), want):
        assert torch.equal(a, b)
    out = store.as_strided((70, 96), (ld, 1), 2048)
    stream = torch.cuda.current_stream().cuda_stream
    eq.add_rms_norm(fx, ld, fr, ld, w, eq.BF16, eq.BF16, 70, 96, 1e-6, 0.0, fr, ld, out, ld, 0, stream)
    assert torch.equal(out, want[0]) and torch.equal(fr, want[1])


@gpu
def test_launch_errors_come_back(monkeypatch):
    x, residual, w = inputs(4, 64, 1, torch.bfloat16, torch.bfloat16, 0.0)
    _, s, f = norm.add_rms_norm(x, residual, w, save=True)
    monkeypatch.setenv("EQUARX_INJECT_LAUNCH_ERROR", "719")
    for call in (lambda: norm.add_rms_norm(x, residual, w), lambda: norm.add_rms_norm_fp8(x, residual, w),
                 lambda: norm.add_rms_norm_backward(x, None, s, f, w), lambda: norm.add_rms_norm_backward(x[:0], None, s[:0], f[:0], w)):
        with pytest.raises(eq.EquarxError) as err:
            call()
        assert err.value.status == binding.ERR_CUDA and eq.last_cuda_error() == 719


@gpu
def test_shapes_that_do_not_fit():
    x, residual, w = inputs(4, 64, 1, torch.bfloat16, torch.bfloat16, 0.0)
    _, s, f = norm.add_rms_norm(x, residual, w, save=True)
    for bad in ((x, residual[:3], w), (x, residual[:, :63], w), (x, residual, w[:63]), (x, residual.half(), w), (x, residual, w.half()),
                (x, residual, w[None]), (x.T, residual.T, w), (x, residual, w.repeat(2)[::2])):
        with pytest.raises(ValueError):
            norm.add_rms_norm(*bad)
        with pytest.raises(ValueError):
            norm.add_rms_norm_fp8(*bad)
    for bad in ((x[:3], None, s, f, w), (x, s[:3], s, f, w), (x, None, s, f[:3], w), (x, None, s, f.half(), w), (x, None, s, f, w[:3])):
        with pytest.raises(ValueError):
            norm.add_rms_norm_backward(*bad)
    with pytest.raises(eq.EquarxError):
        norm.add_rms_norm(x.float(), residual.float(), w.float())              # activations have 16 bits
    with pytest.raises(eq.EquarxError):
        norm.add_rms_norm(x, residual, w, -1.0)
