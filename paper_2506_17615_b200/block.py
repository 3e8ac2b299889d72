"""A tensor-parallel feed-forward block over N simulated ranks, end to end on one GPU.

Each rank holds its slices of the weights.  Serving: the block over 4-bit or 8-bit weights (fp4_gated, then
fp4_linear for the down projection, or their 8-bit forms) gives a bf16 partial sum for each rank, and the quantized AllReduce
adds them.  Training: the block over 16-bit weights with its gradients, from dh, which a library product with the down
projection gives, to dx and the gradients of gate and up; the AllReduce adds the ranks' dx.

serve_layer and train_layer put the residual stream in front: the AllReduce's output of the layer before is added to it and
normalised (norm.add_rms_norm, in 8 bits where the projections take those).  Requests may have low-rank adapters of the down
projection (adapters.add_adapters); the AllReduce then adds the adapters' parts with the rest.

    python -m paper_2506_17615_b200.block --ranks 8 --tokens 512 --hidden 3840 --width 15360 [--format mx|nv|mx8] [--adapters 4]

prints how far the results are from the unsharded block in fp32, and the device time of each part.
"""
import argparse
import json

import torch

from . import adapters, binding, feedforward as ff, norm


class Block:
    """The weights of `ranks` ranks: gate and up [width / ranks, hidden], down [hidden, width / ranks]; the norm's weight, stored
    as its difference from 1, and adapters, if there are any, of the down projection: a [count, rank, width / ranks] for each
    rank, b [count, hidden, rank] and scale [count] for all."""

    NORM_OFFSET = 1.0

    def __init__(self, ranks, hidden, width, act=ff.ACT_GELU_TANH, format=ff.FP4_NV, seed=0, device="cuda"):
        if width % ranks:
            raise ValueError("width must be a multiple of ranks")
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.ranks, self.hidden, self.act = ranks, hidden, act
        f = width // ranks

        def weights(rows, cols, fan_in):
            return [(torch.randn(rows, cols, generator=gen, device=device) * fan_in ** -0.5).bfloat16() for _ in range(ranks)]

        self.gate, self.up, self.down = weights(f, hidden, hidden), weights(f, hidden, hidden), weights(hidden, f, width)
        self.eight = format == ff.FP8_MX
        quantize = ff.fp8_quantize if self.eight else lambda w: ff.fp4_quantize(w, format)
        self.gate4, self.up4, self.down4 = ([quantize(w) for w in ws] for ws in (self.gate, self.up, self.down))
        self.norm = (torch.randn(hidden, generator=gen, device=device) * 0.1).bfloat16()
        self.adapter_a = self.adapter_b = self.adapter_scale = None

    def add_adapters(self, count, rank=16, seed=0):
        """Random adapters of the down projection, for serve_layer's index."""
        gen = torch.Generator(device=self.norm.device)
        gen.manual_seed(seed)

        def normal(*shape, fan_in):
            return (torch.randn(*shape, generator=gen, device=self.norm.device) * fan_in ** -0.5).bfloat16()

        f = self.down[0].shape[1]
        self.adapter_a = [normal(count, rank, f, fan_in=f * self.ranks) for _ in range(self.ranks)]
        self.adapter_b = normal(count, self.hidden, rank, fan_in=rank)
        self.adapter_scale = torch.rand(count, generator=gen, device=self.norm.device) + 0.5

    def allreduce(self, partials, block=256):
        """The quantized AllReduce of the ranks' [tokens, hidden] partial sums, in place."""
        n, count = self.ranks, partials[0].numel()
        if count % (n * block):
            raise ValueError(f"tokens * hidden must be a multiple of {n * block}")
        nbytes = binding.allreduce_sim_pipelined_workspace_bytes(n, count, block)
        ws = partials[0].new_empty(nbytes, dtype=torch.uint8)
        stream = torch.cuda.current_stream(partials[0].device).cuda_stream
        binding.allreduce_sim_pipelined(partials, partials, n, count, block, ws, nbytes, False, stream)
        return partials

    def partials(self, x, index=None):
        """Serving: the ranks' partial sums, everything in 4 or 8 bits (x: a matrix in 16, or in 8 bits an Fp8Matrix), and with
        the adapter of each token that has one in index (int32 [tokens])."""
        if self.eight and not isinstance(x, ff.Fp8Matrix):
            x = ff.fp8_quantize(x)
        gated, linear = (ff.fp8_gated, ff.fp8_linear) if self.eight else (ff.fp4_gated, ff.fp4_linear)
        sums = []
        for r, (g, u, d) in enumerate(zip(self.gate4, self.up4, self.down4)):
            h = gated(x, g, u, self.act)
            y = linear(h, d)
            if index is not None:
                adapters.add_adapters(y, h, self.adapter_a[r], self.adapter_b, index, self.adapter_scale, out=y)
            sums.append(y)
        return sums

    def serve(self, x):
        return self.allreduce(self.partials(x))[0]

    def serve_layer(self, x, residual, index=None):
        """(the AllReduce's output, the residual stream) from those of the layer before."""
        forward = norm.add_rms_norm_fp8 if self.eight else norm.add_rms_norm
        y, total = forward(x, residual, self.norm, offset=self.NORM_OFFSET)
        return self.allreduce(self.partials(y, index))[0], total

    def train_partials(self, x, dy):
        """Training: for each rank its dx and the gradients of its gate and up weights."""
        grads = []
        for wg, wu, wd in zip(self.gate, self.up, self.down):
            h, g, u = ff.gated_forward(x, wg, wu, self.act, save=True)
            grads.append(ff.gated_backward(torch.mm(dy, wd), x, wg, wu, g, u, self.act))
        return grads

    def train(self, x, dy):
        grads = self.train_partials(x, dy)
        dx = self.allreduce([dx for dx, _, _ in grads])[0]
        return dx, [dwg for _, dwg, _ in grads], [dwu for _, _, dwu in grads]


    def train_layer(self, x, residual, dy, dsum):
        """From the gradients of the layer's output and of its residual stream: (d of x and residual, dnorm, dwg, dwu)."""
        y, total, factors = norm.add_rms_norm(x, residual, self.norm, offset=self.NORM_OFFSET, save=True)
        dx, dwg, dwu = self.train(y, dy)
        dstream, dnorm = norm.add_rms_norm_backward(dx, dsum, total, factors, self.norm, self.NORM_OFFSET)
        return dstream, dnorm, dwg, dwu


def layer_reference(block, x, residual, dy, dsum, index=None):
    """(y, sum, d of x and residual, dnorm) of the unsharded layer in fp32; gradients without the adapters"""
    total = (x.float() + residual.float()).requires_grad_()
    weight = block.norm.float().requires_grad_()
    n = total * torch.rsqrt(total.square().mean(1, keepdim=True) + 1e-6) * (weight + block.NORM_OFFSET)
    wg, wu, wd = torch.cat(block.gate).float(), torch.cat(block.up).float(), torch.cat(block.down, dim=1).float()
    g = n @ wg.t()
    h = (torch.nn.functional.silu(g) if block.act == ff.ACT_SILU else torch.nn.functional.gelu(g, approximate="tanh")) * (n @ wu.t())
    y = h @ wd.t()
    ((y * dy.float()).sum() + (total * dsum.float()).sum()).backward()
    y = y.detach()
    if index is not None:
        a = torch.cat(block.adapter_a, dim=2).float()
        for i in range(a.shape[0]):
            rows = (index == i).nonzero()[:, 0]
            y[rows] += block.adapter_scale[i] * (h.detach()[rows] @ a[i].t()) @ block.adapter_b[i].float().t()
    return y, total.detach(), total.grad, weight.grad


def reference(block, x, dy):
    """(y, dx) of the unsharded block in fp32"""
    wg, wu = (torch.cat(w).float() for w in (block.gate, block.up))
    wd = torch.cat(block.down, dim=1).float()
    xr = x.float().requires_grad_()
    g = xr @ wg.t()
    a = torch.nn.functional.silu(g) if block.act == ff.ACT_SILU else torch.nn.functional.gelu(g, approximate="tanh")
    y = (a * (xr @ wu.t())) @ wd.t()
    y.backward(dy.float())
    return y.detach(), xr.grad


def device_us(fn, steps):
    fn()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    start.record()
    for _ in range(steps):
        fn()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) * 1e3 / steps


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--ranks", type=int, default=8)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--hidden", type=int, default=3840)
    p.add_argument("--width", type=int, default=15360, help="of all ranks together")
    p.add_argument("--format", choices=("mx", "nv", "mx8"), default="nv")
    p.add_argument("--adapters", type=int, default=0, help="requests with an adapter each; one more has none")
    p.add_argument("--act", choices=("gelu", "silu"), default="gelu")
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args(argv)
    block = Block(a.ranks, a.hidden, a.width, {"gelu": ff.ACT_GELU_TANH, "silu": ff.ACT_SILU}[a.act],
                  {"mx": ff.FP4_MX, "nv": ff.FP4_NV, "mx8": ff.FP8_MX}[a.format])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, dy = (torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16() for _ in range(2))
    y, (dx, _, _) = block.serve(x), block.train(x, dy)
    y_ref, dx_ref = reference(block, x, dy)
    residual, dsum = (torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16() for _ in range(2))
    index = None
    if a.adapters:
        block.add_adapters(a.adapters)
        index = (torch.arange(a.tokens, device="cuda") * (a.adapters + 1) // a.tokens - 1).int()
    out, _ = block.serve_layer(x, residual, index)
    dstream, _, _, _ = block.train_layer(x, residual, dy, dsum)
    out_ref, _, dstream_ref, _ = layer_reference(block, x, residual, dy, dsum, index)
    ff.check()
    rel = lambda got, want: float((got.float() - want).norm() / want.norm())
    parts = block.partials(x)
    print(json.dumps({
        "ranks": a.ranks, "tokens": a.tokens, "hidden": a.hidden, "width": a.width, "format": a.format,
        "serve_rel_error": round(rel(y, y_ref), 4), "train_dx_rel_error": round(rel(dx, dx_ref), 4),
        "serve_layer_rel_error": round(rel(out, out_ref), 4), "train_layer_rel_error": round(rel(dstream, dstream_ref), 4),
        "us": {f"partials_{8 if block.eight else 4}bit_all_ranks": round(device_us(lambda: block.partials(x), a.steps), 1),
               "allreduce": round(device_us(lambda: block.allreduce(parts), a.steps), 1),
               "train_all_ranks": round(device_us(lambda: block.train(x, dy), a.steps), 1),
               "serve_layer": round(device_us(lambda: block.serve_layer(x, residual, index), a.steps), 1),
               "train_layer": round(device_us(lambda: block.train_layer(x, residual, dy, dsum), a.steps), 1)}}))


if __name__ == "__main__":
    main()
