"""The feed-forward operators: refusals (no GPU), and the kernels against 64-bit references."""
import math
import os
import subprocess
import sys

import pytest
import torch

import ff_reference as ref
import paper_2506_17615_b200 as eq
from paper_2506_17615_b200 import binding
from paper_2506_17615_b200 import feedforward as ff

A = 0x7000_0000_0000          # a made-up, well aligned "device address"
GB = 1 << 30
gpu = pytest.mark.gpu
FORMATS = [eq.FP4_MX, eq.FP4_NV]
ACTS = [eq.ACT_SILU, eq.ACT_GELU_TANH]


def status_of(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except eq.EquarxError as e:
        return e.status
    return 0


# ------------------------------------------------------------------ refusals, sizes (no GPU)

def quantize_args():
    return dict(x=A, dtype=eq.BF16, rows=4, cols=64, ld=64, format=eq.FP4_NV, codes=A + GB, scales=A + 2 * GB,
                row_scales=A + 3 * GB)


def test_quantize_refuses_bad_arguments():
    f, a = eq.fp4_quantize, quantize_args()
    for key in ("x", "codes", "scales", "row_scales"):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**a, key: a[key] + 1}) == binding.ERR_ALIGN
    for key in ("codes", "scales", "row_scales"):
        assert status_of(f, **{**a, key: a[key] + 8}) == binding.ERR_ALIGN
    for key, bad in (("dtype", 3), ("dtype", -1), ("format", 2), ("format", -1)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_FORMAT
    for key, bad in (("cols", 0), ("ld", 63), ("rows", GB + 1), ("cols", GB + 1), ("ld", GB + 1)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
    assert status_of(f, **{**a, "codes": A + 496}) == binding.ERR_ALIAS          # inside x's last row
    assert status_of(f, **{**a, "scales": A + GB + 112}) == binding.ERR_ALIAS    # inside codes
    assert status_of(f, **{**a, "rows": 0, "x": 0, "codes": 0}) == 0             # nothing to do


def test_dequantize_refuses_bad_arguments():
    f = eq.fp4_dequantize
    a = dict(codes=A, scales=A + GB, row_scales=A + 2 * GB, rows=4, cols=64, format=eq.FP4_NV, out=A + 3 * GB,
             dtype=eq.FP32, ld=64)
    for key in ("codes", "scales", "row_scales", "out"):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**a, key: a[key] + 2}) == binding.ERR_ALIGN
    assert status_of(f, **{**a, "dtype": 9}) == binding.ERR_FORMAT
    assert status_of(f, **{**a, "ld": 60}) == binding.ERR_COUNT
    assert status_of(f, **{**a, "out": A + 112}) == binding.ERR_ALIAS


def test_matmul_refuses_bad_arguments():
    f = eq.fp4_matmul
    a = dict(a_codes=A, a_scales=A + GB, a_row_scales=A + 2 * GB, b_codes=A + 3 * GB, b_scales=A + 4 * GB,
             b_row_scales=A + 5 * GB, m=4, n=8, k=64, format=eq.FP4_NV, out=A + 6 * GB, dtype=eq.FP16, ld=8)
    for key in ("a_codes", "a_scales", "a_row_scales", "b_codes", "b_scales", "b_row_scales", "out"):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**a, key: a[key] + (1 if key == "out" else 8)}) == binding.ERR_ALIGN
    for key, bad in (("n", 0), ("k", 0), ("ld", 7), ("m", GB + 1)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
    for key, bad in (("dtype", 3), ("format", 5)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_FORMAT
    assert status_of(f, **{**a, "out": A + 3 * GB + 16}) == binding.ERR_ALIAS
    assert status_of(f, **{**a, "m": 0, "out": 0}) == 0


def test_linear_and_gated_refuse_bad_arguments():
    need = eq.fp4_linear_workspace_bytes(40, 64, eq.FP4_NV)
    w = dict(w_codes=A + GB, w_scales=A + 2 * GB, w_row_scales=A + 3 * GB)
    a = dict(x=A, dtype=eq.BF16, ldx=64, **w, m=40, n=8, k=64, format=eq.FP4_NV, out=A + 4 * GB, ld=8, workspace=A + 5 * GB,
             workspace_bytes=need)
    gu = dict(g_codes=A + GB, g_scales=A + 2 * GB, g_row_scales=A + 3 * GB, u_codes=A + 6 * GB, u_scales=A + 7 * GB,
              u_row_scales=A + 8 * GB)
    b = dict(x=A, dtype=eq.BF16, ldx=64, **gu, m=40, f=8, k=64, format=eq.FP4_NV, act=0, h=A + 4 * GB, ldh=8,
             workspace=A + 5 * GB, workspace_bytes=need)
    for f, args, out in ((eq.fp4_linear, a, "out"), (eq.fp4_gated, b, "h")):
        pointers = [k for k in args if isinstance(args[k], int) and args[k] >= A]
        assert len(pointers) == (6 if f is eq.fp4_linear else 9)
        for key in pointers:
            assert status_of(f, **{**args, key: 0}) == binding.ERR_NULL
            assert status_of(f, **{**args, key: args[key] + (1 if key in ("x", out) else 8)}) == binding.ERR_ALIGN
        assert status_of(f, **{**args, "workspace_bytes": need - 1}) == binding.ERR_WORKSPACE
        assert status_of(f, **{**args, "dtype": eq.FP32}) == binding.ERR_FORMAT     # activations are 16-bit
        assert status_of(f, **{**args, "ldx": 32}) == binding.ERR_COUNT
        assert status_of(f, **{**args, out: A + 5 * GB}) == binding.ERR_ALIAS       # the workspace
        assert status_of(f, **{**args, "m": 0}) == 0
    assert status_of(eq.fp4_gated, **{**b, "act": 2}) == binding.ERR_FORMAT
    assert eq.fp4_linear_workspace_bytes(1, 64, eq.FP4_NV) == 0       # a few tokens are quantized by the product


def test_gated_forward_and_backward_refuse_bad_arguments():
    fwd = dict(x=A, ldx=64, wg=A + GB, ldwg=64, wu=A + 2 * GB, ldwu=64, dtype=eq.FP16, m=4, f=8, k=64, act=1, h=A + 3 * GB,
               ldh=8, g=A + 4 * GB, u=A + 5 * GB, ldgu=8, workspace=0, workspace_bytes=0)
    f = eq.gated_forward
    for key in ("x", "wg", "wu", "h", "g", "u"):
        assert status_of(f, **{**fwd, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**fwd, "workspace": A + 9 * GB, "workspace_bytes": GB, key: fwd[key] + 1}) == binding.ERR_ALIGN
    for key, bad in (("f", 0), ("k", 0), ("ldx", 63), ("ldwg", 63), ("ldwu", 63), ("ldh", 7), ("ldgu", 7)):
        assert status_of(f, **{**fwd, key: bad}) == binding.ERR_COUNT
    for key, bad in (("dtype", eq.FP32), ("act", 2)):
        assert status_of(f, **{**fwd, key: bad}) == binding.ERR_FORMAT
    assert status_of(f, **{**fwd, "h": A + GB}) == binding.ERR_ALIAS
    assert status_of(f, **{**fwd, "ldx": 65}) == binding.ERR_NULL                 # now a workspace is needed
    assert status_of(f, **{**fwd, "ldx": 65, "workspace": A + 9 * GB}) == binding.ERR_WORKSPACE

    need = eq.gated_backward_workspace_bytes(4, 8, 64, A, 64, A, 64, A, 64)
    bwd = dict(dh=A, lddh=8, x=A + GB, ldx=64, wg=A + 2 * GB, ldwg=64, wu=A + 3 * GB, ldwu=64, g=A + 4 * GB, u=A + 5 * GB,
               ldgu=8, dtype=eq.BF16, m=4, f=8, k=64, act=0, dx=A + 6 * GB, lddx=64, dwg=A + 7 * GB, lddwg=64,
               dwu=A + 8 * GB, lddwu=64, workspace=A + 9 * GB, workspace_bytes=need)
    f = eq.gated_backward
    for key in ("dh", "x", "wg", "wu", "g", "u", "dx", "dwg", "dwu", "workspace"):
        assert status_of(f, **{**bwd, key: 0}) == binding.ERR_NULL
        assert status_of(f, **{**bwd, "workspace_bytes": GB, key: bwd[key] + (8 if key == "workspace" else 1)}) == binding.ERR_ALIGN
    for key in ("lddh", "ldgu"):
        assert status_of(f, **{**bwd, key: 7}) == binding.ERR_COUNT
    for key in ("ldx", "ldwg", "ldwu", "lddx", "lddwg", "lddwu"):
        assert status_of(f, **{**bwd, key: 63}) == binding.ERR_COUNT
    assert status_of(f, **{**bwd, "workspace_bytes": need - 1}) == binding.ERR_WORKSPACE
    assert status_of(f, **{**bwd, "dx": A + GB}) == binding.ERR_ALIAS             # in place is not allowed
    assert status_of(f, **{**bwd, "dwu": A + 7 * GB}) == binding.ERR_ALIAS
    assert eq.last_cuda_error() == 0


def test_projections_in_fp32_are_checked_as_such():
    fwd = dict(x=A, ldx=64, wg=A + GB, ldwg=64, wu=A + 2 * GB, ldwu=64, dtype=eq.FP16 | eq.KEPT_FP32, m=4, f=8, k=64, act=1,
               h=A + 3 * GB, ldh=8, g=A + 4 * GB, u=A + 5 * GB, ldgu=8, workspace=0, workspace_bytes=0)
    need = eq.gated_backward_workspace_bytes(4, 8, 64, A, 64, A, 64, A, 64)
    bwd = dict(dh=A, lddh=8, x=A + GB, ldx=64, wg=A + 2 * GB, ldwg=64, wu=A + 3 * GB, ldwu=64, g=A + 4 * GB, u=A + 5 * GB,
               ldgu=8, dtype=eq.BF16 | eq.KEPT_FP32, m=4, f=8, k=64, act=0, dx=A + 6 * GB, lddx=64, dwg=A + 7 * GB, lddwg=64,
               dwu=A + 8 * GB, lddwu=64, workspace=A + 9 * GB, workspace_bytes=need)
    for call, args in ((eq.gated_forward, fwd), (eq.gated_backward, bwd)):
        for key in ("g", "u"):
            assert status_of(call, **{**args, key: args[key] + 2}) == binding.ERR_ALIGN
        for bad in (eq.FP32 | eq.KEPT_FP32, 2 * eq.KEPT_FP32, -1):
            assert status_of(call, **{**args, "dtype": bad}) == binding.ERR_FORMAT
    assert status_of(eq.gated_forward, **{**fwd, "u": fwd["g"] + 112}) == binding.ERR_ALIAS      # g is 128 bytes long
    assert status_of(eq.gated_backward, **{**bwd, "dx": bwd["g"] + 112}) == binding.ERR_ALIAS
    assert eq.last_cuda_error() == 0


def side_by_side():
    def forward(g, u, ldgu, h=A + 3 * GB, ldh=8, m=4):
        return status_of(eq.gated_forward, x=A, ldx=64, wg=A + GB, ldwg=64, wu=A + 2 * GB, ldwu=64, dtype=eq.FP16, m=m, f=8, k=64,
                         act=1, h=h, ldh=ldh, g=g, u=u, ldgu=ldgu, workspace=0, workspace_bytes=0)

    far = A + 5 * GB
    for g, u in ((far, far + 16), (far + 16, far), (far, far + 48), (far + 64, far + 16), (far, far + 64 * 5 + 16)):
        assert forward(g, u, 32) == binding.ERR_CUDA, (g - far, u - far)        # rows of 64 bytes, 16 of them used
    for g, u in ((far, far + 14), (far + 14, far), (far, far + 50), (far + 64, far + 14), (far, far), (far, far + 128)):
        assert forward(g, u, 32) == binding.ERR_ALIAS, (g - far, u - far)
    assert forward(far, far + 16, 16) == binding.ERR_CUDA                       # the halves fill the buffer
    assert forward(far, far + 16, 8) == binding.ERR_ALIAS
    # h in the rows of g and u, with their stride or another; a single row lies between rows or not
    assert forward(far, far + 16, 32, far + 32, 32) == binding.ERR_CUDA
    assert forward(far, far + 16, 32, far + 40, 24) == binding.ERR_ALIAS
    assert forward(far, far + 16, 32, far + 16, 32) == binding.ERR_ALIAS
    one = dict(dtype=eq.BF16, rows=1, cols=8, ld=8, format=eq.FP4_MX, codes=far + 2 * GB, scales=A + GB, row_scales=0)
    assert status_of(eq.fp4_quantize, x=far + 2 * GB + 16, **one) == binding.ERR_CUDA
    assert status_of(eq.fp4_quantize, x=far + 2 * GB + 14, **one) == binding.ERR_ALIAS


def test_matrices_side_by_side_are_no_overlap():
    """Columns of one buffer are accepted, shared elements are not.  What is accepted stops at an injected launch error,
    which the library remembers, so this runs in a process of its own; no launch reaches a GPU."""
    here = os.path.dirname(os.path.abspath(__file__))
    paths = os.pathsep.join([here, os.path.dirname(here)])
    child = subprocess.run([sys.executable, "-c", "import test_feedforward as t; t.side_by_side()"], capture_output=True, text=True,
                           env={**os.environ, "PYTHONPATH": paths, "EQUARX_INJECT_LAUNCH_ERROR": "719"}, timeout=300)
    assert child.returncode == 0, child.stderr


def test_sizes_of_the_buffers():
    assert eq.fp4_codes_bytes(3, 33) == 3 * 32                    # two groups of 32 codes
    assert eq.fp4_scales_bytes(1, 1, eq.FP4_MX) == 1024           # one stage of 256 columns, 128 rows, 8 scales each
    assert eq.fp4_scales_bytes(129, 257, eq.FP4_NV) == 2 * 2 * 2048
    assert eq.fp4_scales_bytes(0, 64, eq.FP4_NV) == 0 and eq.fp4_codes_bytes(4, 0) == 0
    assert eq.fp4_scales_bytes(4, 64, 7) == 0
    assert eq.gated_forward_workspace_bytes(8, 16, 64, A, 64, A, 72, A, 80) == 0
    assert eq.gated_forward_workspace_bytes(8, 16, 64, A, 65, A, 64, A, 64) == 8 * 64 * 2        # x is copied
    assert eq.gated_forward_workspace_bytes(8, 16, 64, A, 64, A, 64, A + 2, 64) == 16 * 64 * 2   # wu is
    assert eq.gated_forward_workspace_bytes(8, 16, 64, A, 63, A, 64, A, 64) == 0                 # invalid


def test_tensors_that_do_not_fit_are_refused():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ff.fp4_quantize(x)                                        # not on a GPU
    with pytest.raises(ValueError):
        ff.gated_forward(x, x, x)


def test_what_the_extension_module_refuses():
    """before any CUDA call: what is no tensor, no matrix, not on a GPU, or the wrong number of arguments"""
    cpu = torch.zeros(4, 8, dtype=torch.bfloat16)
    q = ff.Fp4Matrix(torch.zeros(16, dtype=torch.uint8), 4, 8, eq.FP4_NV)
    for call in (lambda: ff.fp4_quantize(None), lambda: ff.fp4_linear([1], q), lambda: ff.gated_forward(cpu, cpu, 3),
                 lambda: ff._native.quantize(cpu), lambda: ff._native.linear(), lambda: ff.fp4_quantize(cpu, "nv")):
        with pytest.raises((TypeError, ValueError)):
            call()
    for call in (lambda: ff.fp4_quantize(cpu[0]), lambda: ff.fp4_dequantize(q), lambda: ff.fp4_dequantize(q, torch.float64),
                 lambda: ff.fp4_matmul(q, q), lambda: ff.gated_backward(cpu, cpu, cpu, cpu, cpu, cpu),
                 lambda: ff._native.bind("nothing", A)):
        with pytest.raises(ValueError):
            call()


def test_the_module_belongs_to_the_installed_torch(monkeypatch):
    """another torch, however old its files, makes the extension module stale"""
    from paper_2506_17615_b200 import _build
    assert not _build.torch_module_stale()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "1.0")
        assert _build.torch_module_stale()
    with monkeypatch.context() as m:
        m.setattr(_build, "torch_stamp", lambda: "")
        assert _build.torch_module_stale()
    assert not _build.torch_module_stale()


# ------------------------------------------------------------------ inputs

def normal(rows, cols, seed, dtype, scale=1.0, pad=0):
    gen = torch.Generator().manual_seed(seed)
    t = (torch.randn(rows, cols + pad, generator=gen) * scale).to(dtype).cuda()
    return t[:, :cols]


def hard_rows(cols, dtype):
    """rows where a quantiser can go wrong: zeros, ties, range ends, one element alone, subnormals"""
    gen = torch.Generator().manual_seed(5)
    top = torch.finfo(dtype).max
    rows = [torch.zeros(cols), torch.full((cols,), top), torch.full((cols,), torch.finfo(dtype).tiny / 4)]
    ties = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    for scale in (1.0, 2.0 ** -9, 3.0, 2.0 ** 7):
        t = (ties * scale).repeat(-(-cols // 16))[:cols]
        rows += [t, -t, t.flip(0)]
    alone = torch.zeros(cols)
    alone[cols // 2] = -1e-3
    rows.append(alone)
    rows.append(torch.randn(cols, generator=gen) * torch.exp2(torch.randint(-12, 9, (cols,), generator=gen).float()))
    wild = torch.randn(cols, generator=gen) * torch.exp2(torch.arange(cols) / cols * 20 - 10)
    rows.append(wild)
    if dtype != torch.float16:
        rows += [torch.randn(cols, generator=gen) * 2.0 ** -104, torch.randn(cols, generator=gen) * 2.0 ** -99,
                 torch.randn(cols, generator=gen) * 2.0 ** 120, torch.full((cols,), 2.0 ** -127), torch.full((cols,), 2.0 ** -100)]
    return torch.stack(rows).clamp(-top, top).to(dtype).cuda()


# ------------------------------------------------------------------ 4-bit quantisation

def check_quantized(x, fmt):
    q = ff.fp4_quantize(x, fmt)
    rows, cols = x.shape
    code, neg, byte, d, g = ref.quantize(x.double(), fmt)
    stride = -(-cols // 32) * 16
    assert q.codes.shape == (rows, stride)
    nib = torch.stack([q.codes & 15, q.codes >> 4], -1).reshape(rows, -1).long()
    flat = code.reshape(rows, -1)
    want = torch.zeros(rows, stride * 2, dtype=torch.long, device=x.device)
    n = min(flat.shape[1], want.shape[1])
    want[:, :n] = flat[:, :n]
    assert torch.equal(nib & 7, want), "magnitudes differ"
    signs = torch.zeros_like(want, dtype=torch.bool)
    signs[:, :n] = neg.reshape(rows, -1)[:, :n]
    wrong = ((nib >> 3).bool() != signs) & (want > 0)            # the sign of a zero code is free
    assert not bool(wrong.any()), "signs differ"
    pos = ref.scale_positions(rows, byte.shape[1], cols, fmt).to(x.device)
    assert torch.equal(q.scales[pos].long(), byte.long()), "scales differ"
    if fmt == eq.FP4_NV:
        assert torch.equal(q.row_scales.double(), g)
    # scale bytes past the last column, up to the stage's end, are zero
    per = 8 if fmt == eq.FP4_MX else 16
    total = -(-cols // 256) * per
    if total > byte.shape[1]:
        tail = ref.scale_positions(rows, total, cols, fmt)[:, byte.shape[1]:].to(x.device)
        assert not bool(q.scales[tail].any())
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        back = ff.fp4_dequantize(q, dtype)
        assert torch.equal(back.double(), ref.f32(ref.values(x.double(), fmt)).to(dtype).double()), dtype
    ff.check()


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 16, 0), (3, 17, 0), (5, 31, 2), (128, 256, 0), (129, 257, 7),
                                           (33, 500, 12), (1, 5376, 0), (1300, 96, 0), (1200, 1001, 0), (300, 2050, 6),
                                           (2, 24576, 0), (3, 30001, 0)])
def test_quantize_matches_the_definition(fmt, dtype, rows, cols, pad):
    check_quantized(normal(rows, cols, rows + cols, dtype, 3.0, pad), fmt)


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("cols", [16, 64, 333, 512])
def test_quantize_hard_rows(fmt, dtype, cols):
    check_quantized(hard_rows(cols, dtype), fmt)


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_not_finite_elements_become_nan(fmt):
    x = normal(6, 96, 1, torch.bfloat16)
    x[1, 40], x[3, 0], x[4, 95] = float("inf"), float("nan"), float("-inf")
    back = ff.fp4_dequantize(ff.fp4_quantize(x, fmt), torch.float32)
    block = 32 if fmt == eq.FP4_MX else 96
    nan = torch.zeros(6, 96, dtype=torch.bool, device="cuda")
    for r, c in ((1, 40), (3, 0), (4, 95)):
        nan[r, c // block * block:(c // block + 1) * block] = True
    assert torch.equal(back.isnan(), nan)
    w = ff.fp4_quantize(normal(40, 96, 2, torch.bfloat16), fmt)
    for y in (ff.fp4_linear(x, w), ff.fp4_linear(x.repeat(40, 1), w)[:6], torch.cat([ff.fp4_linear(t, w) for t in x.split(2)])):
        rows = y.isnan()
        assert bool(rows[[1, 3, 4]].all()) and not bool(rows[[0, 2, 5]].any())


# ------------------------------------------------------------------ products over 4-bit operands

SIZES = [(1, 1, 1), (1, 16, 32), (1, 130, 300), (3, 100, 64), (16, 128, 256), (17, 129, 257), (64, 257, 1000),
         (127, 300, 513), (128, 64, 96), (129, 128, 256), (130, 300, 500), (257, 129, 777), (300, 513, 1030),
         (520, 1000, 2000), (1025, 260, 64), (2, 140, 2049), (8, 700, 1500), (9, 129, 1025), (16, 260, 4100), (128, 300, 5000),
         (64, 520, 3000)]


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_fp4_products(fmt, m, n, k):
    for i, dtype in enumerate((torch.bfloat16, torch.float16)):
        x = normal(m, k, m + n + i, dtype, 1.0, pad=(0, 3, 8)[(m + i) % 3])
        w = normal(n, k, n + k + i, dtype, k ** -0.5)
        wq = ff.fp4_quantize(w, fmt)
        y = ff.fp4_linear(x, wq)
        value, bound = ref.product(ref.values(x.double(), fmt), ref.values(w.double(), fmt))
        assert y.dtype == dtype
        ref.assert_within(y, value, ref.rounded(value, bound, dtype), "linear")
        xq = ff.fp4_quantize(x, fmt)
        assert torch.equal(ff.fp4_matmul(xq, wq, dtype), y)                       # the same product
        y32 = ff.fp4_matmul(xq, wq, torch.float32)
        ref.assert_within(y32, value, ref.rounded(value, bound, torch.float32), "matmul, fp32")
    ff.check()


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,f,k", SIZES)
def test_fp4_gated(fmt, act, m, f, k):
    dtype = torch.bfloat16 if (m + f) % 2 else torch.float16
    x = normal(m, k, m + f, dtype, 1.0, pad=(0, 1, 8)[m % 3])
    wg, wu = normal(f, k, f + 1, dtype, 2 * k ** -0.5), normal(f, k, f + 2, dtype, k ** -0.5)
    h = ff.fp4_gated(x, ff.fp4_quantize(wg, fmt), ff.fp4_quantize(wu, fmt), act)
    value, bound, _, _ = ref.gated(*(ref.values(t.double(), fmt) for t in (x, wg, wu)), act)
    ref.assert_within(h, value, ref.rounded(value, bound, dtype), "h")
    ff.check()


# (tokens, outputs, columns) of products with more tiles than the 74 pairs of SMs, so that a pair hands accumulators over from
# one tile to the next.  In order: 187 tiles of 256 outputs, the last ones of 40 outputs (one group of 128 scales) and
# of 4 tokens (the pair's second CTA has none); 264 tiles, outputs that TMA cannot write; 79 tiles of 128 outputs.
MANY = [(4100, 2600, 700), (6000, 2587, 300), (20000, 100, 500)]


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,n,k", MANY)
def test_fp4_products_of_many_tiles(fmt, m, n, k):
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        source = torch.bfloat16 if dtype == torch.float32 else dtype
        x, w = normal(m, k, 1, source), normal(n, k, 2, source, k ** -0.5)
        xq, wq = ff.fp4_quantize(x, fmt), ff.fp4_quantize(w, fmt)
        y = ff.fp4_matmul(xq, wq, dtype)
        value, bound = ref.product(ref.values(x.double(), fmt), ref.values(w.double(), fmt))
        ref.assert_within(y, value, ref.rounded(value, bound, dtype), "matmul")
        # the same bits as products of few tokens, in which no pair has a second tile
        for first in range(0, m, 1000):
            assert torch.equal(ff.fp4_matmul(ff.fp4_quantize(x[first:first + 1000], fmt), wq, dtype), y[first:first + 1000])
    ff.check()


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,f,k", [(4100, 1300, 700), (6000, 1293, 300), (20000, 70, 500)])
def test_fp4_gated_of_many_tiles(fmt, m, f, k):
    dtype = torch.bfloat16
    x, wg, wu = normal(m, k, 1, dtype), normal(f, k, 2, dtype, 2 * k ** -0.5), normal(f, k, 3, dtype, k ** -0.5)
    qg, qu = ff.fp4_quantize(wg, fmt), ff.fp4_quantize(wu, fmt)
    h = ff.fp4_gated(x, qg, qu)
    value, bound, _, _ = ref.gated(*(ref.values(t.double(), fmt) for t in (x, wg, wu)), eq.ACT_GELU_TANH)
    ref.assert_within(h, value, ref.rounded(value, bound, dtype), "h")
    for first in range(0, m, 1000):
        assert torch.equal(ff.fp4_gated(x[first:first + 1000], qg, qu), h[first:first + 1000])
    ff.check()


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("parts", range(1, 9))
def test_few_tokens_on_every_cluster_size(fmt, parts):
    """A product of one tile of features over `parts` stages of 256 columns runs on a cluster of `parts` CTAs, each
    with one stage of x.  The row's largest element lies in each CTA's part in turn: every CTA has to know it."""
    dtype, f = torch.bfloat16, 100
    for k in (256 * parts, 256 * parts - 77):
        wg, wu = normal(f, k, k + 1, dtype, 2 * k ** -0.5), normal(f, k, k + 2, dtype, k ** -0.5)
        qg, qu = ff.fp4_quantize(wg, fmt), ff.fp4_quantize(wu, fmt)
        vg, vu = ref.values(wg.double(), fmt), ref.values(wu.double(), fmt)
        for m in (1, 2):
            for part in range(parts):
                x = normal(m, k, part, dtype)
                # the tokens' peaks in this part and, for the second token, in the one before
                for row in range(m):
                    x[row, (part - row) % parts * 256 + 3 + 170 * (part & 1)] = 60.0 + row
                vx = ref.values(x.double(), fmt)
                value, bound = ref.product(vx, vg)
                want, limit, _, _ = ref.gated(vx, vg, vu, eq.ACT_SILU)
                first, gated = ff.fp4_linear(x, qg), ff.fp4_gated(x, qg, qu, eq.ACT_SILU)
                ref.assert_within(first, value, ref.rounded(value, bound, dtype), "linear")
                ref.assert_within(gated, want, ref.rounded(want, limit, dtype), "gated")
                for _ in range(5):
                    assert torch.equal(ff.fp4_linear(x, qg), first) and torch.equal(ff.fp4_gated(x, qg, qu, eq.ACT_SILU), gated)
    ff.check()


# ------------------------------------------------------------------ 16-bit block and its gradients

def backward_reference(dh, x, wg, wu, g, u, act, unit):
    """gradients from the saved g and u, and bounds: dG and dU carry one 16-bit rounding each"""
    a, s = ref.act(g, act), ref.slope(g, act)
    du, dg = dh * a, dh * u * s
    # fp32 evaluation: the slope is a sum of terms up to 1 + |g| in size
    edu = (unit + 2.0 ** -18) * du.abs() + ref.TINY[torch.float16]
    edg = unit * dg.abs() + (2.0 ** -18) * (dh * u).abs() * (1 + g.abs()) + ref.TINY[torch.float16]
    f, m = wg.shape[0], x.shape[0]
    dx = dg @ wg + du @ wu
    acc = 2 * f * ref.ACC
    ex = (edg + acc * dg.abs()) @ wg.abs() + (edu + acc * du.abs()) @ wu.abs()
    dwg, dwu = dg.T @ x, du.T @ x
    ewg = (edg + m * ref.ACC * dg.abs()).T @ x.abs()
    ewu = (edu + m * ref.ACC * du.abs()).T @ x.abs()
    return (dx, ex), (dwg, ewg), (dwu, ewu)


TRAIN = [(1, 1, 1), (1, 64, 64), (2, 130, 72), (16, 128, 256), (33, 65, 129), (128, 200, 300), (129, 256, 128),
         (200, 77, 1001), (257, 300, 513), (512, 520, 264), (1030, 128, 200), (128, 256, 3000), (4100, 100, 136), (2100, 130, 65),
         (100, 1500, 96)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,f,k", TRAIN)
def test_gated_forward_and_backward(dtype, act, m, f, k):
    pad = (0, 8, 3)[(m + f) % 3]
    x = normal(m, k, m + f, dtype, 1.0, pad)
    wg, wu = normal(f, k, f + 1, dtype, 2 * k ** -0.5, pad), normal(f, k, f + 2, dtype, k ** -0.5, (0, 5)[k % 2])
    dh = normal(m, f, m + 3, dtype, 1.0, pad)
    h, g, u = ff.gated_forward(x, wg, wu, act, save=True)
    xd, wgd, wud, dhd = (t.double() for t in (x, wg, wu, dh))
    value, bound, (gv, eg), (uv, eu) = ref.gated(xd, wgd, wud, act)
    ref.assert_within(h, value, ref.rounded(value, bound, dtype), "h")
    ref.assert_within(g, gv, ref.rounded(gv, eg, dtype), "g")
    ref.assert_within(u, uv, ref.rounded(uv, eu, dtype), "u")
    assert torch.equal(ff.gated_forward(x, wg, wu, act), h)
    grads = ff.gated_backward(dh, x, wg, wu, g, u, act)
    want = backward_reference(dhd, xd, wgd, wud, g.double(), u.double(), act, ref.UNIT[dtype])
    for name, got, (v, e) in zip(("dx", "dwg", "dwu"), grads, want):
        assert got.dtype == dtype
        ref.assert_within(got, v, ref.rounded(v, e, dtype), name)
    again = ff.gated_backward(dh, x, wg, wu, g, u, act)
    assert all(torch.equal(p, q) for p, q in zip(grads, again)), "not deterministic"
    ff.check()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,f,k", [(4100, 1300, 1400), (2500, 1501, 1300), (20000, 30, 200)])
def test_gated_forward_and_backward_of_many_tiles(dtype, m, f, k):
    """More tiles than the 74 pairs of SMs: forward 187, 120 and 79; backward 202 and 142 of dx and the weights'
    gradients in one launch, and 79 of dx beside weights' gradients that are split over the tokens."""
    act = eq.ACT_GELU_TANH
    x, wg, wu = normal(m, k, 1, dtype), normal(f, k, 2, dtype, 2 * k ** -0.5), normal(f, k, 3, dtype, k ** -0.5)
    dh = normal(m, f, 4, dtype)
    h, g, u = ff.gated_forward(x, wg, wu, act, save=True)
    xd, wgd, wud, dhd = (t.double() for t in (x, wg, wu, dh))
    value, bound, (gv, eg), (uv, eu) = ref.gated(xd, wgd, wud, act)
    ref.assert_within(h, value, ref.rounded(value, bound, dtype), "h")
    ref.assert_within(g, gv, ref.rounded(gv, eg, dtype), "g")
    ref.assert_within(u, uv, ref.rounded(uv, eu, dtype), "u")
    for first in range(0, m, 1000):
        assert torch.equal(ff.gated_forward(x[first:first + 1000], wg, wu, act), h[first:first + 1000])
    grads = ff.gated_backward(dh, x, wg, wu, g, u, act)
    for name, got, (v, e) in zip(("dx", "dwg", "dwu"), grads,
                                 backward_reference(dhd, xd, wgd, wud, g.double(), u.double(), act, ref.UNIT[dtype])):
        ref.assert_within(got, v, ref.rounded(v, e, dtype), name)
    assert all(torch.equal(p, q) for p, q in zip(grads, ff.gated_backward(dh, x, wg, wu, g, u, act)))
    ff.check()


@gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,f,k", [(5, 40, 24), (150, 96, 136)])
def test_gradients_against_differences(act, m, f, k):
    """<gradient, v> against a central difference of the 64-bit block along v.  The difference's own error
    is O(step^2) of the third derivative (below 1e-6 here); the gradient's is its bound summed along |v|,
    with g and u off by their 16-bit rounding as well."""
    dtype = torch.float16
    x, wg, wu = normal(m, k, 1, dtype), normal(f, k, 2, dtype, k ** -0.5), normal(f, k, 3, dtype, k ** -0.5)
    dh = normal(m, f, 4, dtype)
    _, g, u = ff.gated_forward(x, wg, wu, act, save=True)
    grads = ff.gated_backward(dh, x, wg, wu, g, u, act)
    args = [t.double() for t in (x, wg, wu)]
    unit = ref.UNIT[dtype]

    def loss(x, wg, wu):
        return (dh.double() * ref.act(x @ wg.T, act) * (x @ wu.T)).sum()

    # slopes change by at most 1.2 times the change of g (the second derivatives stay below 1.2)
    bounds = backward_reference(dh.double(), *args, g.double(), u.double(), act, unit)
    eg, eu = unit * g.double().abs(), unit * u.double().abs()
    s = ref.slope(g.double(), act).abs()
    ddg = dh.double().abs() * (eu * (s + 1.2 * eg) + u.double().abs() * 1.2 * eg)
    ddu = dh.double().abs() * 1.2 * eg
    moved = (ddg @ args[1].abs() + ddu @ args[2].abs(), ddg.T @ args[0].abs(), ddu.T @ args[0].abs())
    for i, (got, (v, e), extra) in enumerate(zip(grads, bounds, moved)):
        gen = torch.Generator().manual_seed(10 + i)
        direction = torch.randn(got.shape, generator=gen, dtype=torch.float64).cuda()
        step = 1e-4
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + step * direction, args[i] - step * direction
        numeric = (loss(*plus) - loss(*minus)) / (2 * step)
        tol = ((ref.rounded(v, e, dtype) + extra) * direction.abs()).sum() + 1e-5 * numeric.abs() + 1e-6
        assert abs(float((got.double() * direction).sum() - numeric)) <= float(tol), i


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,f,k", TRAIN + [(4100, 1300, 200)])
def test_projections_kept_in_fp32(dtype, act, m, f, k):
    pad = (0, 8, 3)[(m + f) % 3]
    x = normal(m, k, m + f, dtype, 1.0, pad)
    wg, wu = normal(f, k, f + 1, dtype, 2 * k ** -0.5, pad), normal(f, k, f + 2, dtype, k ** -0.5, (0, 5)[k % 2])
    dh = normal(m, f, m + 3, dtype, 1.0, pad)
    h, g, u = ff.gated_forward(x, wg, wu, act, save=torch.float32)
    assert g.dtype == u.dtype == torch.float32 and torch.equal(ff.gated_forward(x, wg, wu, act), h)
    xd, wgd, wud, dhd = (t.double() for t in (x, wg, wu, dh))
    (gv, eg), (uv, eu) = ref.product(xd, wgd), ref.product(xd, wud)
    ref.assert_within(g, gv, ref.rounded(gv, eg, torch.float32), "g")
    ref.assert_within(u, uv, ref.rounded(uv, eu, torch.float32), "u")
    grads = ff.gated_backward(dh, x, wg, wu, g, u, act)
    want = backward_reference(dhd, xd, wgd, wud, g.double(), u.double(), act, ref.UNIT[dtype])
    for name, got, (v, e) in zip(("dx", "dwg", "dwu"), grads, want):
        assert got.dtype == dtype
        ref.assert_within(got, v, ref.rounded(v, e, dtype), name)
    # nearer to the gradients of the unrounded projections than with g and u kept in 16 bits
    if min(m, f, k) > 60:
        _, g16, u16 = ff.gated_forward(x, wg, wu, act, save=True)
        off = lambda got, v: float((got.double() - v).norm() / v.norm())
        exact = backward_reference(dhd, xd, wgd, wud, gv, uv, act, ref.UNIT[dtype])
        for near, far, (v, _) in zip(grads, ff.gated_backward(dh, x, wg, wu, g16, u16, act), exact):
            assert off(near, v) < off(far, v)
    ff.check()


@gpu
@pytest.mark.parametrize("extra", [0, 3, 4])
@pytest.mark.parametrize("m,f,k", [(3, 130, 72), (300, 264, 136)])
def test_fp32_projections_in_wider_rows(m, f, k, extra):
    """through the C ABI, g beside u in rows of any stride, the first at any element; the rest keeps its canary"""
    dtype, stream = torch.bfloat16, torch.cuda.current_stream().cuda_stream
    x, wg, wu, dh = normal(m, k, 1, dtype), normal(f, k, 2, dtype), normal(f, k, 3, dtype), normal(m, f, 4, dtype)
    h0, g0, u0 = ff.gated_forward(x, wg, wu, save=torch.float32)
    grads = ff.gated_backward(dh, x, wg, wu, g0, u0)
    ld, kind = 2 * f + extra, eq.BF16 | eq.KEPT_FP32
    store = torch.full(((m + 1) * ld + extra,), -77.0, device="cuda")
    gu = store[extra:].as_strided((m, ld), (ld, 1))
    at = lambda col: gu.data_ptr() + 4 * col
    h = torch.empty_like(h0)
    eq.gated_forward(x, k, wg, k, wu, k, kind, m, f, k, eq.ACT_GELU_TANH, h, f, at(0), at(f), ld, 0, 0, stream)
    assert torch.equal(h, h0) and torch.equal(gu[:, :f], g0) and torch.equal(gu[:, f:2 * f], u0)
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    nb = eq.gated_backward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    eq.gated_backward(dh, f, x, k, wg, k, wu, k, at(0), at(f), ld, kind, m, f, k, eq.ACT_GELU_TANH, dx, k, dwg, k, dwu, k, ws, nb, stream)
    for a, b in zip((dx, dwg, dwu), grads):
        assert torch.equal(a, b)
    gu[:, :2 * f] = -77.0
    assert bool((store == -77.0).all())
    # and through torch tensors that are views of it
    eq.gated_forward(x, k, wg, k, wu, k, kind, m, f, k, eq.ACT_GELU_TANH, h, f, at(0), at(f), ld, 0, 0, stream)
    for a, b in zip(ff.gated_backward(dh, x, wg, wu, gu[:, :f], gu[:, f:2 * f]), grads):
        assert torch.equal(a, b)
    with pytest.raises(ValueError):
        ff.gated_backward(dh, x, wg, wu, g0, u0.to(dtype))
    with pytest.raises(ValueError):
        ff.gated_forward(x, wg, wu, save=torch.float16)
    leaf = x.clone().requires_grad_()
    out = ff.gated_forward(leaf, wg, wu, save=torch.float32)
    out[0].backward(dh)
    assert torch.equal(out[1], g0) and torch.equal(leaf.grad, grads[0])
    ff.check()


@gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("large", [True, False])
@pytest.mark.parametrize("m,f,k", [(1, 64, 64), (2, 130, 72), (128, 200, 300), (200, 77, 1001), (512, 520, 264), (4100, 100, 136),
                                   (700, 5000, 96)])
def test_gradients_of_projections_beyond_the_range(dtype, large, m, f, k):
    """dU and dG above 65504 or deep among fp16's subnormal numbers, while dx, dWg and dWu are within its range.  As
    operands they carry one rounding of their type, after a power of two has brought the largest into [2^14, 2^15)."""
    act = eq.ACT_SILU
    if large:                                                     # u about 20, g near 0, dG about 40000 times normal squared
        x, wg, wu = normal(m, k, 1, dtype, 2.0 ** -9), normal(f, k, 2, dtype, 2.0 ** -9), normal(f, k, 3, dtype, 10240 * k ** -0.5)
        dh = normal(m, f, 4, torch.float32, 4000.0).clamp(-60000, 60000).to(dtype)
    else:                                                         # u about 2^-3, dG about 2^-22
        x, wg, wu = normal(m, k, 1, dtype, 2.0 ** 5), normal(f, k, 2, dtype, 2.0 ** -5 * k ** -0.5), \
            normal(f, k, 3, dtype, 2.0 ** -8 * k ** -0.5)
        dh = normal(m, f, 4, dtype, 2.0 ** -18)
    _, g, u = ff.gated_forward(x, wg, wu, act, save=True)
    assert bool(g.isfinite().all()) and bool(u.isfinite().all())
    grads = ff.gated_backward(dh, x, wg, wu, g, u, act)
    x, wg, wu, dh, g, u = (t.double() for t in (x, wg, wu, dh, g, u))
    du, dg = dh * ref.act(g, act), dh * u * ref.slope(g, act)
    if large and m * f > 100:
        assert float(dg.abs().max()) > 65520
    floor, top = 0.0, max(float(du.abs().max()), float(dg.abs().max()))
    if dtype == torch.float16:                                     # half a step of its subnormal numbers, scaled with the rest
        floor = 2.0 ** -25 * (1.0 if 2.0 ** -4 <= top < 65520 else 2.0 ** (math.floor(math.log2(top)) - 14))
    # fp32 evaluation as in backward_reference
    edu = (ref.UNIT[dtype] + 2.0 ** -18) * du.abs() + floor
    edg = ref.UNIT[dtype] * dg.abs() + 2.0 ** -18 * (dh * u).abs() * (1 + g.abs()) + floor
    want = ((dg @ wg + du @ wu, (edg + 2 * f * ref.ACC * dg.abs()) @ wg.abs() + (edu + 2 * f * ref.ACC * du.abs()) @ wu.abs()),
            (dg.T @ x, (edg + m * ref.ACC * dg.abs()).T @ x.abs()), (du.T @ x, (edu + m * ref.ACC * du.abs()).T @ x.abs()))
    for name, got, (v, e) in zip(("dx", "dwg", "dwu"), grads, want):
        ref.assert_within(got, v, ref.rounded(v, e, dtype), name)
    ff.check()


@gpu
@pytest.mark.parametrize("m", [9, 300])
def test_not_finite_gradients_do_not_set_the_range(m):
    """fp16: one token's dh is infinite, another's is NaN; the others' dG above 65504 still give a finite dx"""
    dtype, f, k = torch.float16, 64, 72
    x, wg, wu = normal(m, k, 1, dtype, 2.0 ** -9), normal(f, k, 2, dtype, 2.0 ** -9), normal(f, k, 3, dtype, 10240 * k ** -0.5)
    dh = normal(m, f, 4, torch.float32, 4000.0).clamp(-60000, 60000).to(dtype)
    dh[[2, 4]] = 0.0
    dh[2, 5], dh[4, 0] = float("inf"), float("nan")
    _, g, u = ff.gated_forward(x, wg, wu, save=True)
    dx, dwg, _ = ff.gated_backward(dh, x, wg, wu, g, u)
    rows = [r for r in range(m) if r not in (2, 4)]
    clean, _, _ = ff.gated_backward(dh[rows], x[rows], wg, wu, g[rows], u[rows])
    assert bool(clean.isfinite().all()) and torch.equal(dx[rows], clean)
    assert not bool(dx[[2, 4]].isfinite().any()) and not bool(dwg[[0, 5]].isfinite().any()) and bool(dwg[1].isfinite().all())


def leaves(*tensors):
    return [t.detach().clone().requires_grad_() for t in tensors]


@gpu
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("m", [5, 300])
def test_autograd_connects_forward_and_backward(m, save):
    dtype = torch.bfloat16
    x, wg, wu, dh = normal(m, 72, 1, dtype), normal(40, 72, 2, dtype, 0.1), normal(40, 72, 3, dtype, 0.1), normal(m, 40, 4, dtype)
    h, g, u = ff.gated_forward(x, wg, wu, eq.ACT_SILU, save=True)

    def run(args):
        out = ff.gated_forward(*args, eq.ACT_SILU, save)
        if save:
            assert torch.equal(out[1], g) and torch.equal(out[2], u) and not out[1].requires_grad and not out[2].requires_grad
            out = out[0]
        assert torch.equal(out, h) and out.requires_grad
        return out

    args = leaves(x, wg, wu)
    run(args).backward(dh)
    for t, want in zip(args, ff.gated_backward(dh, x, wg, wu, g, u, eq.ACT_SILU)):
        assert torch.equal(t.grad, want)
    # a gradient that is one element expanded, and one whose columns are not neighbours
    for grad in (torch.ones(1, 1, dtype=dtype, device="cuda").expand(m, 40), dh.T.contiguous().T):
        args = leaves(x, wg, wu)
        run(args).backward(grad)
        for t, want in zip(args, ff.gated_backward(grad.contiguous(), x, wg, wu, g, u, eq.ACT_SILU)):
            assert torch.equal(t.grad, want)
    # only one of the three asks, in the middle of a graph
    for i in range(3):
        args = [x, wg, wu]
        args[i] = leaf = args[i].clone().requires_grad_()
        inner = list(args)
        inner[i] = leaf * 1
        (run(inner) * 2).backward(dh)
        assert torch.equal(leaf.grad, ff.gated_backward(dh * 2, x, wg, wu, g, u, eq.ACT_SILU)[i])
    with torch.no_grad():
        out = ff.gated_forward(*args, eq.ACT_SILU)
        assert torch.equal(out, h) and not out.requires_grad


@gpu
def test_gradients_that_do_not_exist_are_refused():
    dtype = torch.bfloat16
    x, w = normal(4, 64, 1, dtype), normal(8, 64, 2, dtype)
    q = ff.fp4_quantize(w.clone().requires_grad_())                # bytes: nothing to connect
    asking = x.clone().requires_grad_()
    for call in (lambda: ff.fp4_linear(asking, q), lambda: ff.fp4_gated(asking, q, q)):
        with pytest.raises(ValueError, match="no_grad"):
            call()
        with torch.no_grad():
            call()
    assert torch.equal(ff.fp4_linear(asking.detach(), q), ff.fp4_linear(x, q))
    leaf = x.clone().requires_grad_()
    grad, = torch.autograd.grad(ff.gated_forward(leaf, w, w).float().square().sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):                              # no second derivatives
        grad.float().sum().backward()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, x)
        for call in (lambda: ff.gated_forward(dual, w, w), lambda: ff.gated_forward(x, w, torch.autograd.forward_ad.make_dual(w, w)),
                     lambda: ff.fp4_linear(dual, q)):
            with pytest.raises(ValueError, match="tangent"):
                call()


# ------------------------------------------------------------------ no tokens, streams, not finite, guards

@gpu
def test_no_tokens():
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = normal(40, 64, 1, torch.bfloat16)
    for fmt in FORMATS:
        wq = ff.fp4_quantize(w, fmt)
        assert ff.fp4_linear(x, wq).shape == (0, 40) and ff.fp4_gated(x, wq, wq).shape == (0, 40)
        assert ff.fp4_dequantize(ff.fp4_quantize(x, fmt)).shape == (0, 64)
    h, g, u = ff.gated_forward(x, w, w, save=True)
    assert h.shape == (0, 40)
    dx, dwg, dwu = ff.gated_backward(h, x, w, w, g, u)
    assert dx.shape == (0, 64) and not bool(dwg.any()) and not bool(dwu.any())    # sums over nothing


@gpu
def test_on_a_stream_of_its_own():
    """inputs made on one stream, used on another that waits for it; the outputs are the same bits"""
    x, wg, wu = normal(300, 200, 1, torch.bfloat16), normal(256, 200, 2, torch.bfloat16, 0.1), normal(256, 200, 3, torch.bfloat16, 0.1)
    want = ff.gated_forward(x, wg, wu)
    q = ff.fp4_quantize(wg)
    want4 = ff.fp4_linear(x, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = [ff.gated_forward(x * 1, wg, wu) for _ in range(3)]
        y4 = [ff.fp4_linear(x * 1, q) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, want) for t in y) and all(torch.equal(t, want4) for t in y4)


@gpu
@pytest.mark.parametrize("m", [7, 200])
def test_not_finite_values_stay_in_their_rows(m):
    x, wg, wu = normal(m, 100, 1, torch.float16), normal(70, 100, 2, torch.float16, 0.1), normal(70, 100, 3, torch.float16, 0.1)
    clean = ff.gated_forward(x, wg, wu)
    dirty = x.clone()
    dirty[3, 99], dirty[5, 0] = float("nan"), float("inf")
    h, g, u = ff.gated_forward(dirty, wg, wu, save=True)
    keep = [r for r in range(m) if r not in (3, 5)]
    assert torch.equal(h[keep], clean[keep])
    assert bool(h[3].isnan().all()) and not bool(g[5].isfinite().any())
    dx, _, _ = ff.gated_backward(normal(m, 70, 4, torch.float16), dirty, wg, wu, g, u)
    assert bool(dx[keep].isfinite().all()) and bool(dx[3].isnan().all())


@gpu
@pytest.mark.parametrize("m,f,k", [(3, 130, 70), (129, 130, 260), (140, 33, 8)])
def test_strided_outputs_and_no_writes_outside(m, f, k):
    """through the C ABI, into rows inside wider buffers; everything else keeps its canary"""
    dtype, stream = torch.bfloat16, torch.cuda.current_stream().cuda_stream
    x, wg, wu, dh = normal(m, k, 1, dtype), normal(f, k, 2, dtype), normal(f, k, 3, dtype), normal(m, f, 4, dtype)
    h0, g0, u0 = ff.gated_forward(x, wg, wu, save=True)
    grads0 = ff.gated_backward(dh, x, wg, wu, g0, u0)
    for extra in (8, 3):
        def wide(rows, cols):
            return torch.full((rows + 2, cols + extra), -77.0, dtype=dtype, device="cuda")

        def inner(t):        # the row after the first, so that writes in front show too
            return t.data_ptr() + (0 if t.stride(0) % 8 else 2 * t.stride(0))

        def split(t, rows, cols):
            first = 0 if t.stride(0) % 8 else 1
            body = t[first:first + rows, :cols]
            rest = t.clone()
            rest[first:first + rows, :cols] = -77.0
            assert bool((rest == -77.0).all()), "written outside the output"
            return body

        ph, pg, pu = wide(m, f), wide(m, f), wide(m, f)
        nb = eq.gated_forward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
        ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
        eq.gated_forward(x, k, wg, k, wu, k, eq.BF16, m, f, k, eq.ACT_GELU_TANH, inner(ph), f + extra, inner(pg), inner(pu),
                         f + extra, ws, nb, stream)
        for t, want in ((ph, h0), (pg, g0), (pu, u0)):
            assert torch.equal(split(t, m, f), want)
        px, pwg, pwu = wide(m, k), wide(f, k), wide(f, k)
        nb = eq.gated_backward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        eq.gated_backward(dh, f, x, k, wg, k, wu, k, inner(pg), inner(pu), f + extra, eq.BF16, m, f, k, eq.ACT_GELU_TANH,
                          inner(px), k + extra, inner(pwg), k + extra, inner(pwu), k + extra, ws, nb, stream)
        for t, want, rows in ((px, grads0[0], m), (pwg, grads0[1], f), (pwu, grads0[2], f)):
            assert torch.equal(split(t, rows, k), want)
    ff.check()


@gpu
@pytest.mark.parametrize("m,f,k", [(3, 40, 72), (200, 130, 64), (300, 264, 136)])
def test_outputs_side_by_side_in_one_buffer(m, f, k):
    """through the C ABI: h beside x, g and u, dwg and dwu as the halves of wider rows: the bits of separate buffers"""
    dtype, stream = torch.bfloat16, torch.cuda.current_stream().cuda_stream
    x, wg, wu, dh = normal(m, k, 1, dtype), normal(f, k, 2, dtype), normal(f, k, 3, dtype), normal(m, f, 4, dtype)
    h, g, u = ff.gated_forward(x, wg, wu, save=True)
    grads = ff.gated_backward(dh, x, wg, wu, g, u)
    row, gu, dw = torch.zeros(m, k + f, dtype=dtype, device="cuda"), torch.zeros(m, 2 * f, dtype=dtype, device="cuda"), \
        torch.zeros(f, 2 * k, dtype=dtype, device="cuda")
    row[:, :k] = x
    at = lambda t, col: t.data_ptr() + 2 * col
    nb = max(eq.gated_forward_workspace_bytes(m, f, k, row, k + f, wg, k, wu, k), 16)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    eq.gated_forward(row, k + f, wg, k, wu, k, eq.BF16, m, f, k, eq.ACT_GELU_TANH, at(row, k), k + f, gu, at(gu, f), 2 * f, ws, nb, stream)
    assert torch.equal(row, torch.cat([x, h], 1)) and torch.equal(gu, torch.cat([g, u], 1))
    dx = torch.zeros_like(x)
    nb = eq.gated_backward_workspace_bytes(m, f, k, row, k + f, wg, k, wu, k)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    eq.gated_backward(dh, f, row, k + f, wg, k, wu, k, gu, at(gu, f), 2 * f, eq.BF16, m, f, k, eq.ACT_GELU_TANH, dx, k, dw, 2 * k,
                      at(dw, k), 2 * k, ws, nb, stream)
    assert torch.equal(dx, grads[0]) and torch.equal(dw, torch.cat(grads[1:], 1))
    ff.check()


def padded(rows, cols, dtype, beside=8):
    """(buffer, row stride, view): rows that TMA writes, whose last columns fill no 16 bytes, and what lies beside them"""
    ld = (cols + 7) // 8 * 8 + beside
    store = torch.full((rows, ld), -77.0, dtype=dtype, device="cuda")
    return store, ld, store[:, :cols]


def assert_beside(store, cols):
    assert bool((store[:, cols:] == -77.0).all())


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("beside", [0, 8])
@pytest.mark.parametrize("m,f,k", [(3, 33, 75), (300, 130, 101), (261, 5, 67), (1500, 541, 259), (2100, 1663, 126)])
def test_what_lies_beside_an_output_stays(dtype, beside, m, f, k):
    """through the C ABI: the bits of dense outputs, and nothing past an output's last column, whose row goes on to a multiple of 16 bytes"""
    code, stream = {torch.bfloat16: eq.BF16, torch.float16: eq.FP16}[dtype], torch.cuda.current_stream().cuda_stream
    x, wg, wu, dh = normal(m, k, 1, dtype), normal(f, k, 2, dtype, 0.1), normal(f, k, 3, dtype, 0.1), normal(m, f, 4, dtype)
    for fmt in FORMATS:
        q, w = ff.fp4_quantize(x, fmt), ff.fp4_quantize(wg, fmt)
        store, ld, view = padded(m, f, dtype, beside)
        eq.fp4_matmul(q.codes, q.scales, q.row_scales, w.codes, w.scales, w.row_scales, m, f, k, fmt, view, code, ld, stream)
        assert torch.equal(view, ff.fp4_matmul(q, w, dtype))
        assert_beside(store, f)
        nb = eq.fp4_linear_workspace_bytes(m, k, fmt)
        ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
        store, ld, view = padded(m, f, dtype, beside)
        eq.fp4_gated(x, code, k, w.codes, w.scales, w.row_scales, w.codes, w.scales, w.row_scales, m, f, k, fmt, eq.ACT_SILU, view, ld, ws, nb,
                     stream)
        assert torch.equal(view, ff.fp4_gated(x, w, w, eq.ACT_SILU))
        assert_beside(store, f)
    h, g, u = ff.gated_forward(x, wg, wu, save=True)
    grads = ff.gated_backward(dh, x, wg, wu, g, u)
    (sh, ldh, vh), (sg, ldg, vg), (su, _, vu) = (padded(m, f, dtype, beside) for _ in range(3))
    nb = eq.gated_forward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    eq.gated_forward(x, k, wg, k, wu, k, code, m, f, k, eq.ACT_GELU_TANH, vh, ldh, vg, vu, ldg, ws, nb, stream)
    for store, view, want in ((sh, vh, h), (sg, vg, g), (su, vu, u)):
        assert torch.equal(view, want)
        assert_beside(store, f)
    nb = eq.gated_backward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    outs = [padded(rows, k, dtype, beside) for rows in (m, f, f)]
    (sx, ldx, vx), (swg, ldw, vwg), (swu, _, vwu) = outs
    eq.gated_backward(dh, f, x, k, wg, k, wu, k, g, u, f, code, m, f, k, eq.ACT_GELU_TANH, vx, ldx, vwg, ldw, vwu, ldw, ws, nb, stream)
    for (store, _, view), want in zip(outs, grads):
        assert torch.equal(view, want)
        assert_beside(store, k)
    # the matrix that begins right after another's last column
    row = torch.zeros(m, (2 * f + 7) // 8 * 8, dtype=dtype, device="cuda")
    at = lambda col: row.data_ptr() + 2 * col
    nb = eq.gated_forward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    eq.gated_forward(x, k, wg, k, wu, k, code, m, f, k, eq.ACT_GELU_TANH, h, f, at(0), at(f), row.shape[1], ws, nb, stream)
    assert torch.equal(row[:, :f], g) and torch.equal(row[:, f:2 * f], u)
    ff.check()


@gpu
@pytest.mark.parametrize("offset", [1, 2, 4, 7])
@pytest.mark.parametrize("m,f,k", [(5, 40, 72), (200, 136, 264)])
def test_views_that_start_anywhere(m, f, k, offset):
    """operands and outputs whose first element lies `offset` elements into a buffer: the bits of aligned ones"""
    dtype = torch.bfloat16

    def shifted(t):
        store = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
        view = store[offset:].view(t.shape)
        return view.copy_(t)

    x, wg, wu, dh = normal(m, k, 1, dtype), normal(f, k, 2, dtype, 0.1), normal(f, k, 3, dtype, 0.1), normal(m, f, 4, dtype)
    h, g, u = ff.gated_forward(x, wg, wu, save=True)
    grads = ff.gated_backward(dh, x, wg, wu, g, u)
    sx, sg, su = shifted(x), shifted(wg), shifted(wu)
    for a, b in zip(ff.gated_forward(sx, sg, su, save=True), (h, g, u)):
        assert torch.equal(a, b)
    for a, b in zip(ff.gated_backward(shifted(dh), sx, sg, su, shifted(g), shifted(u)), grads):
        assert torch.equal(a, b)
    stream = torch.cuda.current_stream().cuda_stream
    ph, px, pg, pu = shifted(torch.zeros_like(h)), shifted(torch.zeros_like(x)), shifted(torch.zeros_like(wg)), shifted(torch.zeros_like(wu))
    eq.gated_forward(x, k, wg, k, wu, k, eq.BF16, m, f, k, eq.ACT_GELU_TANH, ph, f, 0, 0, 0, 0, 0, stream)
    assert torch.equal(ph, h)
    nb = eq.gated_backward_workspace_bytes(m, f, k, x, k, wg, k, wu, k)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    eq.gated_backward(dh, f, x, k, wg, k, wu, k, g, u, f, eq.BF16, m, f, k, eq.ACT_GELU_TANH, px, k, pg, k, pu, k, ws, nb, stream)
    for a, b in zip((px, pg, pu), grads):
        assert torch.equal(a, b)
    for fmt in FORMATS:
        q, sq = ff.fp4_quantize(x, fmt), ff.fp4_quantize(sx, fmt)
        for out in (torch.bfloat16, torch.float32):
            back = ff.fp4_dequantize(q, out)
            assert torch.equal(back, ff.fp4_dequantize(sq, out))
            pb = shifted(torch.zeros_like(back))
            eq.fp4_dequantize(q.codes, q.scales, q.row_scales, m, k, fmt, pb, {torch.bfloat16: eq.BF16, torch.float32: eq.FP32}[out], k, stream)
            assert torch.equal(pb, back)
            w = ff.fp4_quantize(wg, fmt)
            y = ff.fp4_matmul(q, w, out)
            py = shifted(torch.zeros_like(y))
            eq.fp4_matmul(q.codes, q.scales, q.row_scales, w.codes, w.scales, w.row_scales, m, f, k, fmt, py, {torch.bfloat16: eq.BF16, torch.float32: eq.FP32}[out], f, stream)
            assert torch.equal(py, y)
        w = ff.fp4_quantize(wg, fmt)
        for rows in (1, m):
            assert torch.equal(ff.fp4_linear(sx[:rows], w), ff.fp4_linear(x[:rows], w))
    ff.check()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("cols", [1, 7, 8, 15, 16, 17, 31, 40, 250, 1001, 5002])
def test_quantized_rows_that_start_anywhere(cols, dtype):
    """codes, scales and values of rows at every offset are those of aligned rows; nothing is written beside them"""
    rows, wide = 5, (cols + 31) // 32 * 32 + 32
    code = {torch.bfloat16: eq.BF16, torch.float16: eq.FP16, torch.float32: eq.FP32}[dtype]
    stream = torch.cuda.current_stream().cuda_stream
    gen = torch.Generator(device="cuda").manual_seed(cols)
    aligned = torch.randn(rows, wide, device="cuda", generator=gen).to(dtype)[:, :cols]
    for fmt in FORMATS:
        want = ff.fp4_quantize(aligned, fmt)
        out = torch.empty(rows, wide, device="cuda", dtype=dtype)
        eq.fp4_dequantize(want.codes, want.scales, want.row_scales, rows, cols, fmt, out, code, wide, stream)
        pos = ref.scale_positions(rows, -(-cols // (32 if fmt == eq.FP4_MX else 16)), cols, fmt).cuda()
        for offset in range(16):
            for ld in (cols, cols + 1, cols + 6, wide):
                store = torch.full((offset + rows * ld + 16,), -77.0, device="cuda", dtype=dtype)
                view = store[offset:].as_strided((rows, cols), (ld, 1))
                view.copy_(aligned)
                got = ff.fp4_quantize(view, fmt)
                assert torch.equal(got.codes, want.codes) and torch.equal(got.scales[pos], want.scales[pos])
                if fmt == eq.FP4_NV:
                    assert torch.equal(got.row_scales, want.row_scales)
                store.fill_(-77.0)
                eq.fp4_dequantize(got.codes, got.scales, got.row_scales, rows, cols, fmt, view, code, ld, stream)
                assert torch.equal(view, out[:, :cols])
                view.fill_(-77.0)
                assert bool((store == -77.0).all())
    ff.check()


@gpu
def test_offsets_beyond_32_bits():
    """rows 2^26 elements apart: the last ones lie more than 4 GB (and 2^32 elements) after the first"""
    rows, ld = 70, 1 << 26
    store = torch.empty((rows - 1) * ld + 4096, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((rows, 96), (ld, 1))
    x.copy_(normal(rows, 96, 1, torch.bfloat16))
    w, wu = normal(40, 96, 2, torch.bfloat16), normal(40, 96, 3, torch.bfloat16)
    dense = x.contiguous()
    for fmt in FORMATS:
        q = ff.fp4_quantize(w, fmt)
        assert torch.equal(ff.fp4_linear(x, q), ff.fp4_linear(dense, q))
    h, g, u = ff.gated_forward(dense, w, wu, save=True)
    assert torch.equal(ff.gated_forward(x, w, wu), h)
    for a, b in zip(ff.gated_backward(h, x, w, wu, g, u), ff.gated_backward(h, dense, w, wu, g, u)):
        assert torch.equal(a, b)
    # and outputs that far apart: h beside x, in the same rows
    out = store.as_strided((rows, 40), (ld, 1), 1024)
    stream = torch.cuda.current_stream().cuda_stream
    eq.gated_forward(dense, 96, w, 96, wu, 96, eq.BF16, rows, 40, 96, eq.ACT_GELU_TANH, out.data_ptr(), ld, 0, 0, 0, 0, 0, stream)
    assert torch.equal(out, h)
    q = ff.fp4_quantize(dense)
    eq.fp4_dequantize(q.codes, q.scales, q.row_scales, rows, 96, eq.FP4_NV, store.as_strided((rows, 96), (ld, 1), 2048).data_ptr(), eq.BF16, ld, stream)
    assert torch.equal(store.as_strided((rows, 96), (ld, 1), 2048), ff.fp4_dequantize(q))
    ff.check()


@gpu
def test_the_stride_of_a_single_row_does_not_count():
    """a token cut out of a row of more than 2^30 elements, of an odd length"""
    dtype = torch.bfloat16
    store = torch.empty(1, (1 << 30) + 65, dtype=dtype, device="cuda")
    x = store[:, :72]
    assert x.stride(0) > 1 << 30
    x.copy_(normal(1, 72, 1, dtype))
    dense, wg, wu = x.contiguous(), normal(40, 72, 2, dtype), normal(40, 72, 3, dtype)
    h, g, u = ff.gated_forward(dense, wg, wu, save=True)
    assert torch.equal(ff.gated_forward(x, wg, wu), h)
    for a, b in zip(ff.gated_backward(h, x, wg, wu, g, u), ff.gated_backward(h, dense, wg, wu, g, u)):
        assert torch.equal(a, b)
    for fmt in FORMATS:
        q = ff.fp4_quantize(wg, fmt)
        assert torch.equal(ff.fp4_linear(x, q), ff.fp4_linear(dense, q))
        assert torch.equal(ff.fp4_quantize(x, fmt).codes, ff.fp4_quantize(dense, fmt).codes)


@gpu
def test_results_do_not_depend_on_the_other_tokens():
    """NV and MX: a token's result is the same alone and among others of the same form of the product"""
    w, wu = normal(300, 500, 2, torch.bfloat16), normal(300, 500, 3, torch.bfloat16)
    x = normal(2000, 500, 1, torch.bfloat16)
    for fmt in FORMATS:
        q, qu = ff.fp4_quantize(w, fmt), ff.fp4_quantize(wu, fmt)
        whole = ff.fp4_matmul(ff.fp4_quantize(x, fmt), q, torch.float32)
        some = ff.fp4_matmul(ff.fp4_quantize(x[700:1700], fmt), q, torch.float32)
        assert torch.equal(whole[700:1700], some)
        assert torch.equal(ff.fp4_gated(x, q, qu)[700:1700], ff.fp4_gated(x[700:1700], q, qu))


@gpu
def test_backward_overlaps_nothing_it_must_not():
    """The launches of a backward pass overlap; called back to back on the same buffers, with their outputs
    feeding the next call, they give what separate calls give."""
    x, wg, wu = normal(400, 256, 1, torch.bfloat16), normal(200, 256, 2, torch.bfloat16, 0.1), normal(200, 256, 3, torch.bfloat16, 0.1)

    def steps(sync):
        a, w0, w1, out = x.clone(), wg.clone(), wu.clone(), []
        for _ in range(6):
            h, g, u = ff.gated_forward(a, w0, w1, save=True)
            dx, d0, d1 = ff.gated_backward(h, a, w0, w1, g, u)
            if sync:
                torch.cuda.synchronize()
            out.append((h, dx, d0, d1))
            a, w0, w1 = dx, d0, d1                         # every output is the next call's input
            if sync:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return out

    for p, q in zip(steps(False), steps(True)):
        for s, t in zip(p, q):
            assert torch.equal(s.view(torch.int16), t.view(torch.int16))


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_block_with_the_allreduce(fmt):
    """Four ranks' slices of a block, their partial sums added by the quantized AllReduce: the same bits as
    the CPU oracle gives for these partial sums; close to the unsharded block in 16 bits."""
    import oracle
    from paper_2506_17615_b200 import block as blk, workloads as wl
    ranks, tokens, hidden, width = 4, 96, 256, 1024
    b = blk.Block(ranks, hidden, width, ff.ACT_SILU, fmt, seed=3)
    x, dy = normal(tokens, hidden, 1, torch.bfloat16), normal(tokens, hidden, 2, torch.bfloat16)
    for parts in (b.partials(x), [dx for dx, _, _ in b.train_partials(x, dy)]):
        want = oracle.allreduce(wl.as_u16(torch.stack([p.reshape(-1) for p in parts])), 256)["out"]
        got = b.allreduce([p.clone() for p in parts])
        for r in range(ranks):
            assert (wl.as_u16(got[r].reshape(-1)) == want[r]).all()
    y_ref, dx_ref = blk.reference(b, x, dy)
    dx, dwg, dwu = b.train(x, dy)
    # 4 ranks' bf16 roundings and the AllReduce's int8 steps: each int8 step is at most 1/254 of its block's
    # largest element, about 3 times the block's rms, so 4 steps stay below 4 * 3 / 254 = 0.05 of the norm
    assert float((dx.float() - dx_ref).norm() / dx_ref.norm()) < 0.06
    assert len(dwg) == ranks and all(t.shape == (width // ranks, hidden) for t in dwg + dwu)
    # 4 bits: an element is off by at most a quarter of itself (2^-2, halfway between 1 and 1.5), which
    # bounds each of the three quantised products' relative error by 2 * 0.25
    y = b.serve(x)
    assert float((y.float() - y_ref).norm() / y_ref.norm()) < 0.5
    ff.check()


@gpu
def test_recorded_in_a_cuda_graph():
    x, w = normal(4, 256, 1, torch.bfloat16), ff.fp4_quantize(normal(200, 256, 2, torch.bfloat16))
    wg, wu = normal(64, 256, 3, torch.bfloat16), normal(64, 256, 4, torch.bfloat16)
    big = normal(500, 256, 5, torch.bfloat16)

    def everything():
        h, g, u = ff.gated_forward(big, wg, wu, save=True)
        return (ff.fp4_linear(x, w), ff.fp4_linear(x[:1], w), ff.gated_forward(x, wg, wu), h,
                *ff.gated_backward(h, big, wg, wu, g, u), ff.fp4_dequantize(ff.fp4_quantize(big, eq.FP4_MX)))

    want = everything()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_launch_errors_come_back(monkeypatch):
    x, w = normal(4, 64, 1, torch.bfloat16), normal(8, 64, 2, torch.bfloat16)
    monkeypatch.setenv("EQUARX_INJECT_LAUNCH_ERROR", "719")
    for call in (lambda: ff.fp4_quantize(x), lambda: ff.gated_forward(x, w, w)):
        with pytest.raises(eq.EquarxError) as err:
            call()
        assert err.value.status == binding.ERR_CUDA and eq.last_cuda_error() == 719
    monkeypatch.delenv("EQUARX_INJECT_LAUNCH_ERROR")
    ff.gated_forward(x, w, w)
    ff.check()


@gpu
def test_a_wait_that_runs_out_is_reported_once(monkeypatch):
    """a warp whose wait runs out and one that leaves with it; the context stays usable"""
    x, w = normal(4, 64, 1, torch.bfloat16), normal(8, 64, 2, torch.bfloat16)
    want = ff.gated_forward(x, w, w)
    ff.check()
    monkeypatch.setenv("EQUARX_INJECT_TIMEOUT", "50")             # 0.2 ms
    with pytest.raises(eq.EquarxError) as err:
        ff.check()
    assert err.value.status == binding.ERR_TIMEOUT
    monkeypatch.delenv("EQUARX_INJECT_TIMEOUT")
    ff.check()
    assert torch.equal(ff.gated_forward(x, w, w), want)


@gpu
def test_shapes_that_do_not_fit():
    x, w = normal(4, 64, 1, torch.bfloat16), normal(8, 64, 2, torch.bfloat16)
    for bad in ((x, w, w[:, :63]), (x, w, w[:7]), (x.T, w, w), (x, w, w.to(torch.float16)), (x[0], w, w)):
        with pytest.raises(ValueError):
            ff.gated_forward(*bad)
    mx, nv = ff.fp4_quantize(w, eq.FP4_MX), ff.fp4_quantize(w, eq.FP4_NV)
    with pytest.raises(ValueError):
        ff.fp4_matmul(mx, nv)
    with pytest.raises(ValueError):
        ff.fp4_gated(x, mx, nv)
    with pytest.raises(eq.EquarxError):
        ff.fp4_linear(x.float(), nv)                               # activations are 16-bit
