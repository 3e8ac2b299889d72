"""The feed-forward block in front of the AllReduce, for torch tensors.

    h = act(x Wg^T) * (x Wu^T)          gated_forward, fp4_gated
    partial = h Wd^T                    fp4_linear

with 16-bit weights and their gradients (gated_forward, gated_backward), or with weights and
activations in microscaled 4-bit floating point (fp4_quantize, fp4_dequantize, fp4_matmul, fp4_linear,
fp4_gated).  Marshalling only: outputs and workspaces are allocated with torch on the current stream,
the kernels run on it, and every argument check but those on shapes and strides is the library's own
(include/equarx.h has the formulas and layouts).  A failed call raises EquarxError, tensors that do not
fit together raise ValueError; there is no CPU path.

Matrices are [rows, columns] with unit column stride; the row stride is free.
"""
from dataclasses import dataclass

import torch

from . import binding
from .binding import ACT_GELU_TANH, ACT_SILU, FP4_MX, FP4_NV  # noqa: F401  (part of this module's interface)

_DTYPES = {torch.bfloat16: binding.BF16, torch.float16: binding.FP16, torch.float32: binding.FP32}


@dataclass(frozen=True)
class Fp4Matrix:
    """A rows x cols matrix in microscaled 4-bit floating point (FP4_MX or FP4_NV)."""
    codes: torch.Tensor                  # uint8 [rows, ceil(cols/32)*16]
    scales: torch.Tensor                 # uint8, in the tiled order of include/equarx.h
    row_scales: torch.Tensor | None      # float32 [rows] (FP4_NV)
    rows: int
    cols: int
    format: int


def _matrix(t, what, rows=None, cols=None, dtype=None):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be a matrix whose columns are contiguous")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{what} is {tuple(t.shape)}, expected ({rows}, {cols})")
    if t.dtype not in _DTYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{what} has type {t.dtype}")
    return t


def _ld(t):
    # torch reports an arbitrary row stride for a single row
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _stream(t):
    return torch.cuda.current_stream(t.device).cuda_stream


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _on(t):
    """The library launches on the current device: make it the tensor's own."""
    return torch.cuda.device(t.device)


def fp4_quantize(x, format=FP4_NV):
    """x [rows, cols], bfloat16, float16 or float32 -> Fp4Matrix."""
    _matrix(x, "x")
    rows, cols = x.shape
    codes = torch.empty((rows, -(-cols // 32) * 16), dtype=torch.uint8, device=x.device)
    scales = torch.empty(binding.fp4_scales_bytes(rows, cols, format), dtype=torch.uint8, device=x.device)
    row_scales = torch.empty(rows, dtype=torch.float32, device=x.device) if format == FP4_NV else None
    with _on(x):
        binding.fp4_quantize(x, _DTYPES[x.dtype], rows, cols, _ld(x), format, codes, scales, row_scales, _stream(x))
    return Fp4Matrix(codes, scales, row_scales, rows, cols, format)


def fp4_dequantize(q, dtype=torch.bfloat16):
    """The values that q's codes stand for, rounded once to dtype."""
    out = torch.empty((q.rows, q.cols), dtype=dtype, device=q.codes.device)
    with _on(out):
        binding.fp4_dequantize(q.codes, q.scales, q.row_scales, q.rows, q.cols, q.format, out, _DTYPES[dtype], q.cols,
                               _stream(out))
    return out


def fp4_matmul(a, b, dtype=torch.bfloat16):
    """a b^T of two Fp4Matrix of one format: [a.rows, b.rows]."""
    if a.cols != b.cols or a.format != b.format:
        raise ValueError("the operands differ in columns or format")
    out = torch.empty((a.rows, b.rows), dtype=dtype, device=a.codes.device)
    with _on(out):
        binding.fp4_matmul(a.codes, a.scales, a.row_scales, b.codes, b.scales, b.row_scales, a.rows, b.rows, a.cols, a.format,
                           out, _DTYPES[dtype], b.rows, _stream(out))
    return out


def fp4_linear(x, w):
    """x w^T: x [tokens, k] in 16 bits is quantized in the call, w is an Fp4Matrix [n, k]."""
    _matrix(x, "x", cols=w.cols)
    m = x.shape[0]
    out = torch.empty((m, w.rows), dtype=x.dtype, device=x.device)
    nbytes = binding.fp4_linear_workspace_bytes(m, w.cols, w.format)
    ws = _workspace(nbytes, x.device)
    with _on(x):
        binding.fp4_linear(x, _DTYPES[x.dtype], _ld(x), w.codes, w.scales, w.row_scales, m, w.rows, w.cols, w.format, out,
                           w.rows, ws, nbytes, _stream(x))
    return out


def fp4_gated(x, wg, wu, act=ACT_GELU_TANH):
    """act(x wg^T) * (x wu^T): x [tokens, k] in 16 bits, wg and wu Fp4Matrix [f, k] of one format."""
    if (wg.rows, wg.cols, wg.format) != (wu.rows, wu.cols, wu.format):
        raise ValueError("the two weights differ in shape or format")
    _matrix(x, "x", cols=wg.cols)
    m = x.shape[0]
    h = torch.empty((m, wg.rows), dtype=x.dtype, device=x.device)
    nbytes = binding.fp4_linear_workspace_bytes(m, wg.cols, wg.format)
    ws = _workspace(nbytes, x.device)
    with _on(x):
        binding.fp4_gated(x, _DTYPES[x.dtype], _ld(x), wg.codes, wg.scales, wg.row_scales, wu.codes, wu.scales, wu.row_scales,
                          m, wg.rows, wg.cols, wg.format, act, h, wg.rows, ws, nbytes, _stream(x))
    return h


def gated_forward(x, wg, wu, act=ACT_GELU_TANH, save=False):
    """h = act(x wg^T) * (x wu^T) for x [tokens, k], wg and wu [f, k], all bfloat16 or all float16.
    With save: (h, g, u), where g and u are the two projections that gated_backward needs."""
    _matrix(x, "x")
    m, k = x.shape
    f = wg.shape[0]
    _matrix(wg, "wg", f, k, x.dtype)
    _matrix(wu, "wu", f, k, x.dtype)
    h = torch.empty((m, f), dtype=x.dtype, device=x.device)
    g, u = (torch.empty_like(h), torch.empty_like(h)) if save else (None, None)
    ldx, ldwg, ldwu = _ld(x), _ld(wg), _ld(wu)
    nbytes = binding.gated_forward_workspace_bytes(m, f, k, ldx, ldwg, ldwu)
    ws = _workspace(nbytes, x.device)
    with _on(x):
        binding.gated_forward(x, ldx, wg, ldwg, wu, ldwu, _DTYPES[x.dtype], m, f, k, act, h, f, g, u, f, ws, nbytes,
                              _stream(x))
    return (h, g, u) if save else h


def gated_backward(dh, x, wg, wu, g, u, act=ACT_GELU_TANH):
    """(dx, dwg, dwu) of gated_forward from dh [tokens, f] and the g and u it saved."""
    _matrix(x, "x")
    m, k = x.shape
    f = wg.shape[0]
    for t, what, rows, cols in ((wg, "wg", f, k), (wu, "wu", f, k), (dh, "dh", m, f), (g, "g", m, f), (u, "u", m, f)):
        _matrix(t, what, rows, cols, x.dtype)
    ldgu = _ld(g)
    if _ld(u) != ldgu:
        raise ValueError("g and u have different row strides")
    dx = torch.empty((m, k), dtype=x.dtype, device=x.device)
    dwg, dwu = torch.empty((f, k), dtype=x.dtype, device=x.device), torch.empty((f, k), dtype=x.dtype, device=x.device)
    ldx, ldwg, ldwu = _ld(x), _ld(wg), _ld(wu)
    nbytes = binding.gated_backward_workspace_bytes(m, f, k, ldx, ldwg, ldwu)
    ws = _workspace(nbytes, x.device)
    with _on(x):
        binding.gated_backward(dh, _ld(dh), x, ldx, wg, ldwg, wu, ldwu, g, u, ldgu, _DTYPES[x.dtype], m, f, k, act, dx, k,
                               dwg, k, dwu, k, ws, nbytes, _stream(x))
    return dx, dwg, dwu


def check():
    """Synchronises; raises EquarxError if a kernel of this module gave up a wait (its output is incomplete)."""
    binding.feedforward_check()
