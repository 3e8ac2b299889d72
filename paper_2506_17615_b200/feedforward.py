"""The feed-forward block in front of the AllReduce, for torch tensors.

    h = act(x Wg^T) * (x Wu^T)          gated_forward, fp4_gated
    partial = h Wd^T                    fp4_linear

with 16-bit weights and their gradients (gated_forward, gated_backward), or with weights and
activations in microscaled 4-bit floating point (fp4_quantize, fp4_dequantize, fp4_matmul, fp4_linear,
fp4_gated).  Marshalling only: outputs and workspaces are allocated with torch on the current stream,
the kernels run on it, and every argument check but those on shapes, strides and devices is the library's
own (include/equarx.h has the formulas and layouts).  A failed call raises EquarxError, tensors that do
not fit together raise ValueError; there is no CPU path.

Matrices are [rows, columns] with unit column stride; the row stride is free.  A call for a few tokens is
over in a few microseconds on the GPU, so what it costs on the host counts: one output allocation, one
workspace allocation where one is needed, plain integers into the library.
"""
import ctypes
import importlib
from functools import lru_cache

import torch

from . import _build, binding
from .binding import ACT_GELU_TANH, ACT_SILU, FP4_MX, FP4_NV, EquarxError  # noqa: F401  (part of this module's interface)

_DTYPES = {torch.bfloat16: binding.BF16, torch.float16: binding.FP16, torch.float32: binding.FP32}
_lib = binding.lib

# the entry points, by way of the extension module (csrc/fastcall.c) rather than ctypes
_build.build_fastcall()
_fast = importlib.import_module("._fastcall", __package__)
for _name in ("fp4_quantize", "fp4_dequantize", "fp4_matmul", "fp4_linear", "fp4_gated", "gated_forward", "gated_backward"):
    _fast.bind(_name, ctypes.cast(getattr(_lib, "equarx_" + _name), ctypes.c_void_p).value)

# what a call needs beside its tensors depends on its shape, and on how its rows are aligned
_linear_workspace = lru_cache(maxsize=4096)(_lib.equarx_fp4_linear_workspace_bytes)
_forward_workspace = lru_cache(maxsize=4096)(_lib.equarx_gated_forward_workspace_bytes)
_backward_workspace = lru_cache(maxsize=4096)(_lib.equarx_gated_backward_workspace_bytes)


def _up(n, to):
    return -(-n // to) * to


@lru_cache(maxsize=4096)
def _layout(rows, cols, format):
    """offsets of codes and row factors in the buffer of an Fp4Matrix, and its size; scales come first"""
    row_scales = _up(_lib.equarx_fp4_scales_bytes(rows, cols, format), 256)
    codes = row_scales + (_up(4 * rows, 256) if format == FP4_NV else 0)
    return codes, row_scales, codes + _lib.equarx_fp4_codes_bytes(rows, cols)


class Fp4Matrix:
    """A rows x cols matrix in microscaled 4-bit floating point (FP4_MX or FP4_NV): one buffer that holds
    scales, row factors and codes, each part starting on a multiple of 256 bytes."""
    __slots__ = ("data", "rows", "cols", "format", "_parts")

    def __init__(self, data, rows, cols, format):
        self.data, self.rows, self.cols, self.format = data, rows, cols, format
        base = data.data_ptr()
        codes, row_scales, _ = _layout(rows, cols, format)
        self._parts = (base + codes, base, base + row_scales if format == FP4_NV else 0)

    @staticmethod
    def nbytes(rows, cols, format):
        return _layout(rows, cols, format)[2]

    @property
    def codes(self):
        """uint8 [rows, ceil(cols/32)*16], two codes a byte, the first in the low half"""
        first, _, end = _layout(self.rows, self.cols, self.format)
        return self.data[first:end].view(self.rows, _up(self.cols, 32) // 2)

    @property
    def scales(self):
        """uint8, in the tiled order of include/equarx.h"""
        return self.data[:_lib.equarx_fp4_scales_bytes(self.rows, self.cols, self.format)]

    @property
    def row_scales(self):
        """float32 [rows] (FP4_NV), None (FP4_MX)"""
        if self.format != FP4_NV:
            return None
        first = _layout(self.rows, self.cols, self.format)[1]
        return self.data[first:first + 4 * self.rows].view(torch.float32)


def _matrix(t, what):
    """t's shape, row stride, type and device, after the checks"""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a matrix")
    r, c = t.shape
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{what} must be a CUDA tensor")
    dtype = t.dtype
    if dtype not in _DTYPES:
        raise ValueError(f"{what} has type {dtype}")
    return r, c, _row_stride(t, what, r, c), dtype, dev


def _row_stride(t, what, r, c):
    ld, unit = t.stride()
    if unit != 1 and c > 1:
        raise ValueError(f"{what} must have contiguous columns")
    # torch reports any stride for a single row
    return ld if r > 1 else max(ld, c)


def _fits(t, what, r, c, dtype, dev):
    """t's row stride, where t has to be r x c, of this type and on this device"""
    if t.shape != (r, c) or t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{what} is {tuple(t.shape)} {t.dtype} on device {t.get_device()}, expected ({r}, {c}) {dtype} on {dev}")
    return _row_stride(t, what, r, c)


def _call(device, fn, *args):
    """fn(*args, current stream of the device), with the device current"""
    stream = torch._C._cuda_getCurrentRawStream(device)
    if torch._C._cuda_getDevice() == device:
        status = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            status = fn(*args, stream)
    if status:
        raise EquarxError(status, "equarx_" + fn.__name__)


def _like(t):
    """a contiguous matrix of t's shape and type"""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _workspace(like, nbytes):
    """(tensor to keep until the call has been enqueued, its address)"""
    if not nbytes:
        return None, 0
    ws = like.new_empty(nbytes, dtype=torch.uint8)
    return ws, ws.data_ptr()


def fp4_quantize(x, format=FP4_NV):
    """x [rows, cols], bfloat16, float16 or float32 -> Fp4Matrix."""
    rows, cols, ld, dtype, dev = _matrix(x, "x")
    q = Fp4Matrix(x.new_empty(_layout(rows, cols, format)[2], dtype=torch.uint8), rows, cols, format)
    _call(dev, _fast.fp4_quantize, x.data_ptr(), _DTYPES[dtype], rows, cols, ld, format, *q._parts)
    return q


def fp4_dequantize(q, dtype=torch.bfloat16):
    """The values that q's codes stand for, rounded once to dtype."""
    out = q.data.new_empty((q.rows, q.cols), dtype=dtype)
    _call(out.get_device(), _fast.fp4_dequantize, *q._parts, q.rows, q.cols, q.format, out.data_ptr(), _DTYPES[dtype],
          q.cols)
    return out


def fp4_matmul(a, b, dtype=torch.bfloat16):
    """a b^T of two Fp4Matrix of one format: [a.rows, b.rows]."""
    if a.cols != b.cols or a.format != b.format:
        raise ValueError("the operands differ in columns or format")
    out = a.data.new_empty((a.rows, b.rows), dtype=dtype)
    dev = out.get_device()
    if b.data.get_device() != dev:
        raise ValueError("the operands are on different devices")
    _call(dev, _fast.fp4_matmul, *a._parts, *b._parts, a.rows, b.rows, a.cols, a.format, out.data_ptr(), _DTYPES[dtype],
          b.rows)
    return out


def fp4_linear(x, w):
    """x w^T: x [tokens, k] in 16 bits is quantized in the call, w is an Fp4Matrix [n, k]."""
    m, k, ld, dtype, dev = _matrix(x, "x")
    if k != w.cols or dev != w.data.get_device():
        raise ValueError(f"x has {k} columns on device {dev}, the weight {w.cols} on {w.data.get_device()}")
    out = x.new_empty((m, w.rows))
    nbytes = _linear_workspace(m, k, w.format)
    ws, ptr = _workspace(x, nbytes)
    _call(dev, _fast.fp4_linear, x.data_ptr(), _DTYPES[dtype], ld, *w._parts, m, w.rows, k, w.format, out.data_ptr(),
          w.rows, ptr, nbytes)
    return out


def fp4_gated(x, wg, wu, act=ACT_GELU_TANH):
    """act(x wg^T) * (x wu^T): x [tokens, k] in 16 bits, wg and wu Fp4Matrix [f, k] of one format."""
    if wg.rows != wu.rows or wg.cols != wu.cols or wg.format != wu.format:
        raise ValueError("the two weights differ in shape or format")
    m, k, ld, dtype, dev = _matrix(x, "x")
    if k != wg.cols or dev != wg.data.get_device() or dev != wu.data.get_device():
        raise ValueError(f"x has {k} columns on device {dev}, the weights {wg.cols} on {wg.data.get_device()}, {wu.data.get_device()}")
    h = x.new_empty((m, wg.rows))
    nbytes = _linear_workspace(m, k, wg.format)
    ws, ptr = _workspace(x, nbytes)
    _call(dev, _fast.fp4_gated, x.data_ptr(), _DTYPES[dtype], ld, *wg._parts, *wu._parts, m, wg.rows, k, wg.format,
          act, h.data_ptr(), wg.rows, ptr, nbytes)
    return h


def gated_forward(x, wg, wu, act=ACT_GELU_TANH, save=False):
    """h = act(x wg^T) * (x wu^T) for x [tokens, k], wg and wu [f, k], all bfloat16 or all float16.
    With save: (h, g, u), where g and u are the two projections that gated_backward needs."""
    m, k, ldx, dtype, dev = _matrix(x, "x")
    f = wg.shape[0]
    ldg, ldu = _fits(wg, "wg", f, k, dtype, dev), _fits(wu, "wu", f, k, dtype, dev)
    h = x.new_empty((m, f))
    g = u = None
    if save:
        g, u = torch.empty_like(h), torch.empty_like(h)
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    nbytes = _forward_workspace(m, f, k, xp & 15, ldx, gp & 15, ldg, up & 15, ldu)
    ws, ptr = _workspace(x, nbytes)
    _call(dev, _fast.gated_forward, xp, ldx, gp, ldg, up, ldu, _DTYPES[dtype], m, f, k, act, h.data_ptr(), f, g.data_ptr() if save else 0, u.data_ptr() if save else 0, f, ptr, nbytes)
    return (h, g, u) if save else h


def gated_backward(dh, x, wg, wu, g, u, act=ACT_GELU_TANH):
    """(dx, dwg, dwu) of gated_forward from dh [tokens, f] and the g and u it saved."""
    m, k, ldx, dtype, dev = _matrix(x, "x")
    f = wg.shape[0]
    ldwg, ldwu = _fits(wg, "wg", f, k, dtype, dev), _fits(wu, "wu", f, k, dtype, dev)
    lddh, ldgu = _fits(dh, "dh", m, f, dtype, dev), _fits(g, "g", m, f, dtype, dev)
    if _fits(u, "u", m, f, dtype, dev) != ldgu:
        raise ValueError("g and u have different row strides")
    dx, dwg, dwu = _like(x), _like(wg), _like(wu)
    xp, gp, up = x.data_ptr(), wg.data_ptr(), wu.data_ptr()
    nbytes = _backward_workspace(m, f, k, xp & 15, ldx, gp & 15, ldwg, up & 15, ldwu)
    ws, ptr = _workspace(x, nbytes)
    _call(dev, _fast.gated_backward, dh.data_ptr(), lddh, xp, ldx, gp, ldwg, up, ldwu, g.data_ptr(), u.data_ptr(), ldgu, _DTYPES[dtype], m, f, k, act, dx.data_ptr(), k, dwg.data_ptr(), k, dwu.data_ptr(),
          k, ptr, nbytes)
    return dx, dwg, dwu


def check():
    """Synchronises; raises EquarxError if a kernel of this module gave up a wait (its output is incomplete)."""
    binding.feedforward_check()
