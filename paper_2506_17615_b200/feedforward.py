"""The feed-forward block in front of the AllReduce, for torch tensors.

    h = act(x Wg^T) * (x Wu^T)          gated_forward, fp4_gated
    partial = h Wd^T                    fp4_linear

with 16-bit weights and their gradients (gated_forward, gated_backward), or with weights and
activations in microscaled 4-bit floating point (fp4_quantize, fp4_dequantize, fp4_matmul, fp4_linear,
fp4_gated).  Marshalling only, most of it in an extension module (csrc/feedforward_torch.cpp): outputs and
workspaces are allocated with torch on the current stream, the kernels run on it, and every argument check
but those on shapes, strides, types and devices is the library's own (include/equarx.h has the formulas and
layouts).  A failed call raises EquarxError, tensors that do not fit together raise ValueError; there is no
CPU path.

Matrices are [rows, columns] with unit column stride; the row stride is free.

gated_forward takes part in autograd: called with tensors that require gradients, its h is connected to them by
gated_backward.  The 4-bit products have no gradients and refuse such an x (outside torch.no_grad()); a
quantized matrix is bytes, through which no gradient passes.  gated_backward's results have no gradients themselves.
"""
import ctypes
import importlib

import torch

from . import _build, binding
from .binding import ACT_GELU_TANH, ACT_SILU, FP4_MX, FP4_NV, EquarxError  # noqa: F401  (part of this module's interface)

_DTYPES = {torch.bfloat16: binding.BF16, torch.float16: binding.FP16, torch.float32: binding.FP32}

_build.build_torch_module()
_native = importlib.import_module("._feedforward", __package__)
for _name in ("fp4_codes_bytes", "fp4_scales_bytes", "fp4_quantize", "fp4_dequantize", "fp4_matmul", "fp4_linear_workspace_bytes",
              "fp4_linear", "fp4_gated", "gated_forward_workspace_bytes", "gated_forward", "gated_backward_workspace_bytes",
              "gated_backward"):
    _native.bind(_name, ctypes.cast(getattr(binding.lib, "equarx_" + _name), ctypes.c_void_p).value)


class Fp4Matrix:
    """A rows x cols matrix in microscaled 4-bit floating point (FP4_MX or FP4_NV): one buffer that holds
    scales, row factors and codes, each part starting on a multiple of 256 bytes."""
    __slots__ = ("data", "rows", "cols", "format")

    def __init__(self, data, rows, cols, format):
        self.data, self.rows, self.cols, self.format = data, rows, cols, format

    @property
    def codes(self):
        """uint8 [rows, ceil(cols/32)*16], two codes a byte, the first in the low half"""
        _, first, end = _native.layout(self.rows, self.cols, self.format)
        return self.data[first:end].view(self.rows, (self.cols + 31) // 32 * 16)

    @property
    def scales(self):
        """uint8, in the tiled order of include/equarx.h"""
        return self.data[:binding.fp4_scales_bytes(self.rows, self.cols, self.format)]

    @property
    def row_scales(self):
        """float32 [rows] (FP4_NV), None (FP4_MX)"""
        if self.format != FP4_NV:
            return None
        first = _native.layout(self.rows, self.cols, self.format)[0]
        return self.data[first:first + 4 * self.rows].view(torch.float32)


def _or_raise(result, where):
    """a call's tensors; its status, an integer, raises"""
    if result.__class__ is int:
        raise EquarxError(result, where)
    return result


def _code(dtype):
    try:
        return _DTYPES[dtype]
    except KeyError:
        raise ValueError(f"no output of type {dtype}") from None


def fp4_quantize(x, format=FP4_NV):
    """x [rows, cols], bfloat16, float16 or float32 -> Fp4Matrix."""
    data = _or_raise(_native.quantize(x, format), "equarx_fp4_quantize")
    rows, cols = x.shape
    return Fp4Matrix(data, rows, cols, format)


def fp4_dequantize(q, dtype=torch.bfloat16):
    """The values that q's codes stand for, rounded once to dtype."""
    return _or_raise(_native.dequantize(q.data, q.rows, q.cols, q.format, _code(dtype)), "equarx_fp4_dequantize")


def fp4_matmul(a, b, dtype=torch.bfloat16):
    """a b^T of two Fp4Matrix of one format: [a.rows, b.rows]."""
    if a.cols != b.cols or a.format != b.format:
        raise ValueError("the operands differ in columns or format")
    return _or_raise(_native.matmul(a.data, a.rows, b.data, b.rows, a.cols, a.format, _code(dtype)), "equarx_fp4_matmul")


def fp4_linear(x, w):
    """x w^T: x [tokens, k] in 16 bits is quantized in the call, w is an Fp4Matrix [n, k]."""
    return _or_raise(_native.linear(x, w.data, w.rows, w.cols, w.format), "equarx_fp4_linear")


def fp4_gated(x, wg, wu, act=ACT_GELU_TANH):
    """act(x wg^T) * (x wu^T): x [tokens, k] in 16 bits, wg and wu Fp4Matrix [f, k] of one format."""
    if wg.rows != wu.rows or wg.cols != wu.cols or wg.format != wu.format:
        raise ValueError("the two weights differ in shape or format")
    return _or_raise(_native.gated(x, wg.data, wu.data, wg.rows, wg.cols, wg.format, act), "equarx_fp4_gated")


def gated_forward(x, wg, wu, act=ACT_GELU_TANH, save=False):
    """h = act(x wg^T) * (x wu^T) for x [tokens, k], wg and wu [f, k], all bfloat16 or all float16.
    With save: (h, g, u), where g and u are the two projections that gated_backward needs, of x's type, or with
    save=torch.float32 in fp32, for gradients with less rounding and twice the memory of g and u."""
    wide = save is torch.float32
    if isinstance(save, torch.dtype) and not wide and save is not x.dtype:
        raise ValueError(f"g and u are kept in x's type or in torch.float32, not in {save}")
    result = _native.gated_forward(x, wg, wu, act, save, wide)
    if result is None:                                  # gradients are wanted
        return _Gated.apply(x, wg, wu, act, save)
    return _or_raise(result, "equarx_gated_forward")


def gated_backward(dh, x, wg, wu, g, u, act=ACT_GELU_TANH):
    """(dx, dwg, dwu) of gated_forward from dh [tokens, f] and the g and u it saved, in either type."""
    return _or_raise(_native.gated_backward(dh, x, wg, wu, g, u, act), "equarx_gated_backward")


class _Gated(torch.autograd.Function):
    """gated_forward and gated_backward as a pair of autograd's"""

    @staticmethod
    def forward(ctx, x, wg, wu, act, save):
        h, g, u = gated_forward(x, wg, wu, act, save or True)
        ctx.save_for_backward(x, wg, wu, g, u)
        ctx.act = act
        if not save:
            return h
        ctx.mark_non_differentiable(g, u)
        return h, g, u

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, *_):
        if dh.stride(1) != 1 or dh.stride(0) < dh.shape[1]:     # a sum's gradient is one element, expanded
            dh = dh.contiguous()
        return *gated_backward(dh, *ctx.saved_tensors, ctx.act), None, None


def check():
    """Synchronises; raises EquarxError if a kernel of this module gave up a wait (its output is incomplete)."""
    binding.feedforward_check()
