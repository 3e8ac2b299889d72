"""A tensor-parallel feed-forward block over N simulated ranks, end to end on one GPU.

Each rank holds its slices of the weights.  Serving: the block over 4-bit weights (fp4_gated, then
fp4_linear for the down projection) gives a bf16 partial sum for each rank, and the quantized AllReduce
adds them.  Training: the block over 16-bit weights with its gradients, from dh, which a library product with the down
projection gives, to dx and the gradients of gate and up; the AllReduce adds the ranks' dx.

    python -m paper_2506_17615_b200.block --ranks 8 --tokens 512 --hidden 3840 --width 15360 [--format mx]

prints how far both results are from the unsharded block in fp32, and the device time of each part.
"""
import argparse
import json

import torch

from . import binding, feedforward as ff


class Block:
    """The weights of `ranks` ranks: gate and up [width / ranks, hidden], down [hidden, width / ranks]."""

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
        self.gate4, self.up4, self.down4 = ([ff.fp4_quantize(w, format) for w in ws] for ws in (self.gate, self.up, self.down))

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

    def partials(self, x):
        """Serving: the ranks' partial sums, everything in 4 bits."""
        return [ff.fp4_linear(ff.fp4_gated(x, g, u, self.act), d) for g, u, d in zip(self.gate4, self.up4, self.down4)]

    def serve(self, x):
        return self.allreduce(self.partials(x))[0]

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
    p.add_argument("--format", choices=("mx", "nv"), default="nv")
    p.add_argument("--act", choices=("gelu", "silu"), default="gelu")
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args(argv)
    block = Block(a.ranks, a.hidden, a.width, {"gelu": ff.ACT_GELU_TANH, "silu": ff.ACT_SILU}[a.act],
                  {"mx": ff.FP4_MX, "nv": ff.FP4_NV}[a.format])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, dy = (torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16() for _ in range(2))
    y, (dx, _, _) = block.serve(x), block.train(x, dy)
    y_ref, dx_ref = reference(block, x, dy)
    ff.check()
    rel = lambda got, want: float((got.float() - want).norm() / want.norm())
    parts = block.partials(x)
    print(json.dumps({
        "ranks": a.ranks, "tokens": a.tokens, "hidden": a.hidden, "width": a.width, "format": a.format,
        "serve_rel_error": round(rel(y, y_ref), 4), "train_dx_rel_error": round(rel(dx, dx_ref), 4),
        "us": {"partials_4bit_all_ranks": round(device_us(lambda: block.partials(x), a.steps), 1),
               "allreduce": round(device_us(lambda: block.allreduce(parts), a.steps), 1),
               "train_all_ranks": round(device_us(lambda: block.train(x, dy), a.steps), 1)}}))


if __name__ == "__main__":
    main()
