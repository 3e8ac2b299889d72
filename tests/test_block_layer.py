"""A whole layer: residual stream, norm, block, adapters and the quantized AllReduce together."""
import pytest
import torch

import paper_2506_17615_b200 as eq
from paper_2506_17615_b200 import adapters as ad
from paper_2506_17615_b200 import block as blk
from paper_2506_17615_b200 import feedforward as ff
from paper_2506_17615_b200 import norm
from test_feedforward import normal

gpu = pytest.mark.gpu
FORMATS = [eq.FP4_MX, eq.FP4_NV, ff.FP8_MX]
RANKS, HIDDEN, WIDTH = 4, 256, 1024


def layer(fmt, tokens):
    b = blk.Block(RANKS, HIDDEN, WIDTH, ff.ACT_SILU, fmt, seed=3)
    b.add_adapters(3, 8, seed=4)
    x, residual, dy, dsum = (normal(tokens, HIDDEN, 1 + i, torch.bfloat16) for i in range(4))
    index = (torch.arange(tokens) * 4 // tokens - 1).int().cuda()
    return b, x, residual, dy, dsum, index


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens", [4, 96, 300])
def test_layer_with_the_allreduce(fmt, tokens):
    """The parts called one by one give the layer's bits, the AllReduce those of the CPU oracle; the whole is close to the
    unsharded layer in fp32."""
    import oracle
    from paper_2506_17615_b200 import workloads as wl
    b, x, residual, dy, dsum, index = layer(fmt, tokens)
    y, total = norm.add_rms_norm(x, residual, b.norm, offset=1.0)
    q = norm.add_rms_norm_fp8(x, residual, b.norm, offset=1.0)[0] if fmt == ff.FP8_MX else y
    for idx in (None, index):
        parts = b.partials(q, idx)
        want = oracle.allreduce(wl.as_u16(torch.stack([p.reshape(-1) for p in parts])), 256)["out"]
        out, stream = b.serve_layer(x, residual, idx)
        assert (wl.as_u16(out.reshape(-1)) == want[0]).all() and torch.equal(stream, total)
        if idx is not None:                                        # the adapters are in the partial sums
            gated = (lambda g, u: ff.fp8_gated(q, g, u, b.act)) if fmt == ff.FP8_MX else (lambda g, u: ff.fp4_gated(y, g, u, b.act))
            bare = b.partials(q)
            for r, (g, u) in enumerate(zip(b.gate4, b.up4)):
                assert torch.equal(parts[r], ad.add_adapters(bare[r], gated(g, u), b.adapter_a[r], b.adapter_b, idx, b.adapter_scale))
        ref, _, dref, dnorm_ref = blk.layer_reference(b, x, residual, dy, dsum, idx)
        # Three quantised products, each off by at most 2 * 2^-2 (4 bits) or 2 * 2^-4 (8 bits) of itself, and the AllReduce's 0.05;
        # errors of single elements have either sign, so the norm stays below the first alone
        assert float((out.float() - ref).norm() / ref.norm()) < (0.18 if fmt == ff.FP8_MX else 0.5)
    dstream, dnorm, dwg, dwu = b.train_layer(x, residual, dy, dsum)
    _, total, factors = norm.add_rms_norm(x, residual, b.norm, offset=1.0, save=True)
    dx, wg, wu = b.train(y, dy)
    assert all(torch.equal(s, t) for s, t in zip((dstream, dnorm), norm.add_rms_norm_backward(dx, dsum, total, factors, b.norm, 1.0)))
    assert all(torch.equal(s, t) for s, t in zip(dwg + dwu, wg + wu))
    # 16-bit gradients and the AllReduce's four int8 steps: see test_block_with_the_allreduce
    assert float((dstream.float() - dref).norm() / dref.norm()) < 0.06
    assert float((dnorm.float() - dnorm_ref).norm() / dnorm_ref.norm()) < 0.06
    ff.check()


@gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens", [4, 300])
def test_layer_in_a_cuda_graph(fmt, tokens):
    """a serving step and a training step, recorded, replayed on changed inputs"""
    b, x, residual, dy, dsum, index = layer(fmt, tokens)
    b.serve_layer(x, residual, index), b.train_layer(x, residual, dy, dsum)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        served, trained = b.serve_layer(x, residual, index), b.train_layer(x, residual, dy, dsum)
    for seed in (11, 12):
        x.copy_(normal(tokens, HIDDEN, seed, torch.bfloat16))
        index.copy_(index.flip(0))
        graph.replay()
        want, grads = b.serve_layer(x, residual, index), b.train_layer(x, residual, dy, dsum)
        assert all(torch.equal(s, t) for s, t in zip(served, want))
        assert torch.equal(trained[0], grads[0]) and torch.equal(trained[1], grads[1])
        assert all(torch.equal(s, t) for s, t in zip(trained[2] + trained[3], grads[2] + grads[3]))
    ff.check()


@gpu
def test_layer_through_autograd():
    """norm and gated block as autograd connects them, against the calls one by one"""
    b, x, residual, dy, _, _ = layer(eq.FP4_MX, 96)
    wg, wu = b.gate[0], b.up[0]
    dh = normal(96, WIDTH // RANKS, 9, torch.bfloat16)
    leaves = [t.clone().requires_grad_() for t in (x, residual, b.norm, wg, wu)]
    y, total = norm.add_rms_norm(leaves[0], leaves[1], leaves[2], offset=1.0)
    h = ff.gated_forward(y, leaves[3], leaves[4], b.act)
    torch.autograd.backward([h, total], [dh, dy])
    y, total, factors = norm.add_rms_norm(x, residual, b.norm, offset=1.0, save=True)
    _, g, u = ff.gated_forward(y, wg, wu, b.act, save=True)
    dyy, dwg, dwu = ff.gated_backward(dh, y, wg, wu, g, u, b.act)
    dstream, dnorm = norm.add_rms_norm_backward(dyy, dy, total, factors, b.norm, 1.0)
    for leaf, want in zip(leaves, (dstream, dstream, dnorm, dwg, dwu)):
        assert torch.equal(leaf.grad, want)
