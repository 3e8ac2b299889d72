"""The residual stream between an AllReduce and the next block, for torch tensors.

    sum = x + residual
    y = sum / sqrt(mean(sum^2) + eps) * (offset + weight)      add_rms_norm, add_rms_norm_fp8

with y in 16 bits (and gradients: add_rms_norm_backward, or autograd), or in microscaled 8-bit floating point, ready for the
products fp8_matmul and fp8_gated of the feed-forward block.  Marshalling only; include/equarx.h has the arithmetic.
Matrices are [rows, columns] with unit column stride; weight is [columns], of x's type or float32.  offset is 0, or 1 for
weights stored as differences from 1.  A failed call raises EquarxError, tensors that do not fit together raise
ValueError; there is no CPU path.

add_rms_norm takes part in autograd.  Its 8-bit form has no gradients and refuses inputs that ask for one (outside
torch.no_grad()); add_rms_norm_backward's results have no gradients themselves.  A backward pass that is recorded in a CUDA graph
calls add_rms_norm_backward; autograd's own recording needs what torch asks for there (no graph of the same leaves from outside).
"""
import torch

from .feedforward import Fp8Matrix, _native, _or_raise


def add_rms_norm(x, residual, weight, eps=1e-6, offset=0.0, save=False):
    """(y, sum) for x and residual [rows, columns], bfloat16 or float16; residual None: nothing is added and sum is x.
    With save: (y, sum, factors), where factors (float32 [rows]) is what add_rms_norm_backward needs beside sum."""
    result = _native.add_rms_norm(x, residual, weight, eps, offset, save)
    if result is None:                                  # gradients are wanted
        out = _AddRmsNorm.apply(x, residual, weight, eps, offset)
        y, total, factors = out if residual is not None else (out[0], x, out[1])
        return (y, total, factors) if save else (y, total)
    return _or_raise(result, "equarx_add_rms_norm")


def add_rms_norm_fp8(x, residual, weight, eps=1e-6, offset=0.0):
    """(y, sum) with y as a feedforward.Fp8Matrix, quantized from fp32."""
    data, total = _or_raise(_native.add_rms_norm_fp8(x, residual, weight, eps, offset), "equarx_add_rms_norm_fp8")
    return Fp8Matrix(data, *x.shape), total


def add_rms_norm_backward(dy, dsum, sum, factors, weight, offset=0.0):
    """(dx, dweight) from the gradients of y and of sum (None where sum is not used any further), the sum and the factors that
    add_rms_norm saved.  dx is the gradient of x and of residual alike; dweight has weight's type."""
    return _or_raise(_native.add_rms_norm_backward(dy, dsum, sum, factors, weight, offset), "equarx_add_rms_norm_backward")


def _rows(grad):
    """a gradient as a matrix that the library reads: a sum's gradient is one element, expanded"""
    if grad is not None and (grad.stride(1) != 1 or grad.stride(0) < grad.shape[1]):
        return grad.contiguous()
    return grad


class _AddRmsNorm(torch.autograd.Function):
    """add_rms_norm and add_rms_norm_backward as a pair of autograd's"""

    @staticmethod
    def forward(ctx, x, residual, weight, eps, offset):
        y, total, factors = add_rms_norm(x, residual, weight, eps, offset, save=True)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(total, factors, weight)
        ctx.offset, ctx.added = offset, residual is not None
        ctx.mark_non_differentiable(factors)
        return (y, total, factors) if ctx.added else (y, factors)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, *rest):
        dsum = rest[0] if ctx.added else None
        if dy is None:                                  # only the sum goes on
            return dsum, dsum, None, None, None
        total, factors, weight = ctx.saved_tensors
        dx, dweight = add_rms_norm_backward(_rows(dy), _rows(dsum), total, factors, weight, ctx.offset)
        return dx, dx if ctx.added else None, dweight, None, None
