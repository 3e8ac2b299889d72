"""Low-rank adapters of many requests beside a shared projection, for torch tensors.

    y = fp4_linear(x, w)                                 the projection that all requests share
    y = add_adapters(y, x, a, b, index, scale, out=y)    and each token's own adapter

They are added to a projection that exists as a tensor, such as the down projection.  The gated block multiplies gate and up inside
one kernel and gives out neither before the activation, so adapters of those two do not go through it.

Marshalling only; include/equarx.h has the arithmetic.  A failed call raises EquarxError, tensors that do not fit together
raise ValueError; there is no CPU path.  For serving: there are no gradients, and tensors that ask for one are refused
(outside torch.no_grad()).
"""
from .feedforward import _native, _or_raise


def add_adapters(y, x, a, b, index, scale=None, out=None):
    """y[t] + scale[i] (x[t] a[i]^T) b[i]^T with i = index[t], and y[t] where index[t] is no adapter (negative, say).

    y [tokens, n] and x [tokens, k], both bfloat16 or both float16; a [adapters, rank, k] and b [adapters, n, rank], dense, rank
    at most 128; index int32 [tokens]; scale float32 [adapters], None: 1.  out may be y; writing to it advances its version, as torch's own
    calls in place do."""
    return _or_raise(_native.add_adapters(y, x, a, b, index, scale, out), "equarx_add_adapters")
