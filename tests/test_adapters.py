"""Low-rank adapters of many requests: refusals (no GPU), and the kernel against 64-bit references.

Bounds.  x A^T is a sum of k products in fp32, its value enters the second product with 16 bits at least (off by 2^-17 of itself;
fp16: with 22, after a power of two), which is a sum of rank products in fp32, twice (high and low halves); the scale and the
final addition are one fp32 rounding each, and the result is rounded to 16 bits once.
"""
import pytest
import torch

import ff_reference as ref
import paper_2506_17615_b200 as eq
from paper_2506_17615_b200 import adapters as ad
from paper_2506_17615_b200 import binding
from paper_2506_17615_b200 import feedforward as ff
from test_feedforward import A, GB, assert_beside, normal, padded, status_of

gpu = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


def call_args():
    return dict(y=A, ldy=64, x=A + GB, ldx=32, a=A + 2 * GB, b=A + 3 * GB, index=A + 4 * GB, scale=A + 5 * GB, dtype=eq.BF16, tokens=4, n=64,
                k=32, rank=8, adapters=3, out=A + 6 * GB, ldo=64, workspace=0, workspace_bytes=0)


def test_refuses_bad_arguments():
    f, a = eq.add_adapters, call_args()
    for key in ("y", "x", "a", "b", "index", "out"):
        assert status_of(f, **{**a, key: 0}) == binding.ERR_NULL
    for key in ("y", "x", "a", "b", "index", "scale", "out"):
        assert status_of(f, **{**a, key: a[key] + 1}) == binding.ERR_ALIGN
    for bad in (eq.FP32, -1):
        assert status_of(f, **{**a, "dtype": bad}) == binding.ERR_FORMAT
    for key, bad in (("n", 0), ("k", 0), ("rank", 0), ("rank", 129), ("tokens", GB + 1), ("adapters", GB + 1), ("ldy", 63), ("ldx", 31),
                     ("ldo", 63)):
        assert status_of(f, **{**a, key: bad}) == binding.ERR_COUNT
    for bad in (A + 2, A + GB, A + 2 * GB, A + 3 * GB, A + 4 * GB, A + 5 * GB):
        assert status_of(f, **{**a, "out": bad}) == binding.ERR_ALIAS
    assert status_of(f, **{**a, "out": A, "ldo": 72}) == binding.ERR_ALIAS
    assert status_of(f, **{**a, "tokens": 0, "y": 0}) == 0
    # many tokens go through a workspace
    assert eq.add_adapters_workspace_bytes(4, 64, 32, 8, 3) == 0 and eq.add_adapters_workspace_bytes(10 ** 6, 64, 32, 0, 3) == 0
    need = eq.add_adapters_workspace_bytes(10 ** 5, 64, 32, 17, 3)
    assert need >= 10 ** 5 * 32 * 4
    many = {**a, "tokens": 10 ** 5, "rank": 17, "workspace": A + 7 * GB, "workspace_bytes": need}
    assert status_of(f, **{**many, "workspace": 0}) == binding.ERR_NULL
    assert status_of(f, **{**many, "workspace_bytes": need - 1}) == binding.ERR_WORKSPACE
    assert status_of(f, **{**many, "workspace": A + 7 * GB + 8}) == binding.ERR_ALIGN
    for bad in (A, A + GB, A + 3 * GB, A + 6 * GB):
        assert status_of(f, **{**many, "workspace": bad}) == binding.ERR_ALIAS
    assert eq.last_cuda_error() == 0


def test_what_the_extension_module_refuses():
    y, a = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(1, 2, 8, dtype=torch.bfloat16)
    for call in (lambda: ad.add_adapters(y, y, a, a, torch.zeros(4, dtype=torch.int32)), lambda: ad.add_adapters(None, y, a, a, None),
                 lambda: ad.add_adapters(y[0], y, a, a, y)):
        with pytest.raises((TypeError, ValueError)):
            call()


def inputs(tokens, n, k, rank, count, seed, dtype, pad=0):
    y, x = normal(tokens, n, seed, dtype, 1.0, pad), normal(tokens, k, seed + 1, dtype, 1.0, pad)
    a = normal(count * rank, k, seed + 2, dtype, k ** -0.5).contiguous().view(count, rank, k)
    b = normal(count * n, rank, seed + 3, dtype, rank ** -0.5).contiguous().view(count, n, rank)
    scale = torch.rand(count, generator=torch.Generator().manual_seed(seed)).add(0.5).cuda()
    return y, x, a, b, scale


def patterns(tokens, count, seed):
    """indexes of requests one after the other, of tokens of all requests mixed, and of none"""
    gen = torch.Generator().manual_seed(seed)
    mixed = torch.randint(-1, count, (tokens,), generator=gen)
    mixed[tokens // 2] = count + 5                                  # no adapter either
    return [(torch.arange(tokens) * (count + 1) // tokens - 1).int().cuda(), mixed.int().cuda(), torch.full((tokens,), -1).int().cuda()]


def check(out, y, x, a, b, index, scale):
    dtype, value, bound = y.dtype, y.double().clone(), torch.zeros_like(y, dtype=torch.float64)
    for i in range(a.shape[0]):
        rows = (index == i).nonzero()[:, 0]
        c = 1.0 if scale is None else float(scale[i])
        s, es = ref.product(x[rows].double(), a[i].double())
        es = es + (2.0 ** -17 if dtype == torch.bfloat16 else 2.0 ** -21) * s.abs() + 2.0 ** -24 * s.abs()
        d, ed = ref.product(s, b[i].double())
        value[rows] += c * d
        bound[rows] = c * (2 * ed + es @ b[i].double().abs().T) + 2.0 ** -23 * (value[rows].abs() + c * d.abs())
    ref.assert_within(out, value, ref.rounded(value, bound, dtype), "out")
    bare = (index < 0) | (index >= a.shape[0])
    assert torch.equal(out[bare], y[bare])


# a cluster for each token
SIZES = [(1, 1, 1, 1, 1), (1, 64, 64, 16, 1), (1, 5376, 2688, 16, 3), (2, 33, 40, 8, 2), (3, 130, 72, 5, 3), (16, 128, 256, 16, 4),
         (17, 257, 129, 24, 5), (64, 520, 264, 16, 64), (64, 1000, 1000, 64, 9), (100, 96, 3000, 32, 4), (300, 513, 777, 128, 3),
         (601, 264, 136, 64, 7), (700, 64, 64, 1, 700), (40, 2001, 700, 100, 40), (9, 520, 3000, 128, 2)]
# tiles of tokens, of rows that TMA reads and of others
SIZES += [(1500, 5376, 520, 16, 2), (8192, 640, 72, 8, 3), (5000, 1000, 1000, 64, 2), (3000, 1360, 640, 128, 30), (2000, 2640, 1000, 72, 3),
          (2500, 1001, 777, 16, 4), (4100, 600, 201, 40, 5), (1300, 1032, 777, 100, 3), (1030, 3000, 1000, 32, 300), (2049, 2568, 512, 24, 20),
          (70000, 72, 136, 5, 6), (1111, 2500, 2600, 31, 2), (900, 9000, 128, 16, 3)]
# one chunk of columns, one block of features, clusters of one CTA, two for a tile, adapters that a pass over x does not hold
SIZES += [(1200, 7000, 64, 32, 3), (3000, 8, 3000, 16, 5), (40000, 128, 128, 16, 5), (1400, 5000, 1000, 128, 5), (1025, 4096, 2000, 16, 11),
          (2100, 2000, 640, 64, 9), (20000, 300 * 8, 64, 8, 2)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,k,rank,count", SIZES)
def test_matches_the_definition(dtype, tokens, n, k, rank, count):
    pad = (0, 8, 3)[(tokens + n) % 3]
    y, x, a, b, scale = inputs(tokens, n, k, rank, count, tokens + n, dtype, pad)
    for i, index in enumerate(patterns(tokens, count, tokens)):
        c = scale if i != 1 else None
        out = ad.add_adapters(y, x, a, b, index, c)
        check(out, y, x, a, b, index, c)
        assert torch.equal(ad.add_adapters(y, x, a, b, index, c), out), "not deterministic"
        again = y.clone(memory_format=torch.contiguous_format)
        assert ad.add_adapters(again, x, a, b, index, c, out=again) is again and torch.equal(again, out)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 20, 400, 2001])
def test_not_finite_values_stay_with_their_adapter(dtype, tokens):
    k = 72 if tokens < 1000 else 2600                               # tiles of tokens
    y, x, a, b, scale = inputs(tokens, 136, k, 16, 4, 1, dtype)
    assert (eq.add_adapters_workspace_bytes(tokens, 136, k, 16, 4) > 0) == (tokens > 1000)
    index = (torch.arange(tokens) % 4).int().cuda()
    clean = ad.add_adapters(y, x, a, b, index, scale)
    for bad in (float("nan"), float("inf")):
        a2, b2 = a.clone(), b.clone()
        a2[1, 3, 5], b2[2, 7, 0] = bad, bad
        out = ad.add_adapters(y, x, a2, b2, index, scale)
        rows = (index != 1) & (index != 2)
        assert torch.equal(out[rows], clean[rows])
        assert not bool(out[index == 1].isfinite().any())
        two = index == 2
        assert not bool(out[two][:, 7].isfinite().any())
        others = [c for c in range(136) if c != 7]
        assert torch.equal(out[two][:, others], clean[two][:, others])
        x2 = x.clone()
        x2[tokens // 2, 9] = bad
        out = ad.add_adapters(y, x2, a, b, index, scale)
        keep = torch.arange(tokens, device="cuda") != tokens // 2
        assert torch.equal(out[keep], clean[keep]) and not bool(out[tokens // 2].isfinite().any())
        y2 = y.clone()
        y2[0, 3] = bad
        out = ad.add_adapters(y2, x, a, b, index, scale)
        assert not bool(out[0, 3].isfinite()) and torch.equal(out[1:], clean[1:]) and torch.equal(out[0, 4:], clean[0, 4:])


@gpu
@pytest.mark.parametrize("large", [True, False])
@pytest.mark.parametrize("tokens,n", [(40, 64), (12000, 200), (12000, 201)])
def test_products_beyond_the_range_of_fp16(large, tokens, n):
    """x A^T above 65504 or among fp16's subnormal numbers, with outputs inside its range"""
    y, x, a, b, _ = inputs(tokens, n, 96, 16, 3, 1, torch.float16)
    a, b = (a * 2000, b * 2.0 ** -12) if large else (a * 2.0 ** -9, b * 2.0 ** 3)
    x = x * 200 if large else x * 2.0 ** -10
    index = (torch.arange(tokens) % 4 - 1).int().cuda()
    s = x.double() @ a.double()[0].T
    assert float(s.abs().max()) > 70000 if large else float(s.abs().max()) < 2.0 ** -15
    out = ad.add_adapters(y * 0, x, a, b, index)
    check(out, y * 0, x, a, b, index, None)


# a cluster for each token, tiles of rows that TMA reads, tiles of others
FORMS = [(4, 136, 72), (3000, 1360, 640), (3000, 1001, 777)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rank", [1, 5, 8, 33, 72, 100])
@pytest.mark.parametrize("tokens,n,k", FORMS)
def test_infinite_values_in_adapters_whose_ranks_are_padded(dtype, rank, tokens, n, k):
    """what fills the ranks up multiplies no infinity: with positive adapters an infinite element of x gives the definition's infinities,
    and no NaN"""
    y, x, a, b, _ = inputs(tokens, n, k, rank, 3, 1, dtype)
    a, b = a.abs() + 0.01, b.abs() + 0.01
    assert (eq.add_adapters_workspace_bytes(tokens, n, k, rank, 3) > 0) == (tokens > 1000)
    index = (torch.arange(tokens) % 4 - 1).int().cuda()
    clean = ad.add_adapters(y, x, a, b, index)
    for sign in (1.0, -1.0):
        x2 = x.clone()
        x2[2, 9] = sign * float("inf")
        out = ad.add_adapters(y, x2, a, b, index)
        assert bool((out[2] == sign * float("inf")).all())
        keep = torch.arange(tokens, device="cuda") != 2
        assert torch.equal(out[keep], clean[keep])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,k", FORMS)
def test_sums_at_the_end_of_the_range_of_fp32(dtype, tokens, n, k):
    """a finite S that the 16-bit type's range does not hold, or only after a large power of two: S is the scale itself, and what B
    multiplies it with is 0 or brings it back.  2^-17 of S holds here too: below fp32's end at most 2^-8 of S is left beside the type's
    largest number, and that rounds to 8 bits."""
    top = 3.4e38 if dtype == torch.bfloat16 else 2.0 ** 127
    y, _, _, _, _ = inputs(tokens, n, k, 8, 1, 1, dtype)
    x, a, b = (torch.zeros(s, dtype=dtype, device="cuda") for s in ((tokens, k), (2, 8, k), (2, n, 8)))
    x[:, 0], a[:, 0, 0] = 1.0, 1.0
    small = 2.0 ** -100 if dtype == torch.bfloat16 else 2.0 ** -24
    b[:, 1::2, 0] = small                                            # every other feature
    scale = torch.tensor([top, -top], device="cuda")
    index = (torch.arange(tokens) % 3 - 1).int().cuda()
    out = ad.add_adapters(y, x, a, b, index, scale)
    c = torch.where(index < 0, 0.0, scale[index.clamp(min=0).long()]).double()
    part = c[:, None] * b[0, :, 0].double()[None, :]
    want = y.double() + part
    if dtype == torch.float16:                                       # beyond it, or nothing
        assert torch.equal(out, want.to(dtype))
    else:
        ref.assert_within(out, want, ref.rounded(want, (2.0 ** -17 + 2.0 ** -23) * part.abs() + 2.0 ** -23 * want.abs(), dtype), "out")
    assert torch.equal(out[:, 0::2], y[:, 0::2]) and torch.equal(out[index < 0], y[index < 0])


@gpu
def test_a_result_in_place_is_one_to_torch():
    """writing into a tensor advances its version: what an operation has saved of it is not used afterwards"""
    dtype = torch.bfloat16
    y, x, a, b, scale = inputs(6, 96, 64, 16, 5, 1, dtype)
    index = patterns(6, 5, 3)[0]
    w = torch.ones(96, dtype=dtype, device="cuda").requires_grad_()
    for target in (y, y.clone().requires_grad_()):
        z = (target * w).sum()
        before = target._version
        with torch.no_grad():
            assert ad.add_adapters(target, x, a, b, index, scale, out=target) is target
        assert target._version == before + 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()
    # a view's version is its base's, and nothing else's is touched
    base = torch.empty(6, 192, dtype=dtype, device="cuda")
    versions = base._version, y._version, x._version
    out = ad.add_adapters(y, x, a, b, index, scale, out=base[:, 96:])
    assert (base._version, y._version, x._version) == (versions[0] + 1, *versions[1:]) and out._version == base._version
    before = base._version
    ad.add_adapters(y, x, a, b, index, scale)
    with pytest.raises(eq.EquarxError):
        ad.add_adapters(base[:, :96], x, a, b, index, scale, out=base[:, 8:104])
    assert base._version == before                                   # nothing has been written
    # tensors of inference mode have no version, and torch's rule for them holds
    with torch.inference_mode():
        t = torch.zeros(6, 96, dtype=dtype, device="cuda")
        assert torch.equal(ad.add_adapters(y, x, a, b, index, scale, out=t), ad.add_adapters(y, x, a, b, index, scale))
    with pytest.raises(RuntimeError, match="inference"):
        ad.add_adapters(y, x, a, b, index, scale, out=t)


@gpu
@pytest.mark.parametrize("offset", [1, 2, 4, 8])
@pytest.mark.parametrize("tokens", [3, 150, 50001])
def test_views_that_start_anywhere(tokens, offset):
    """through the C ABI; the rest of the output's buffer keeps its canary.  A cluster for each token gives the bits of aligned
    rows; tiles of rows that TMA cannot read add in another order, which the bound of all results allows"""
    dtype, stream, n, k, rank = torch.bfloat16, torch.cuda.current_stream().cuda_stream, 72, 40, 8
    y, x, a, b, scale = inputs(tokens, n, k, rank, 3, 1, dtype)
    index = patterns(tokens, 3, 2)[1]
    want = ad.add_adapters(y, x, a, b, index, scale)

    def assert_same(out):
        if tokens < 1000:
            assert torch.equal(out, want)
        else:
            check(out, y, x, a, b, index, scale)

    def place(t, ld):
        store = torch.full((offset + t.shape[0] * ld + 16,), -77.0, device="cuda", dtype=dtype)
        view = store[offset:].as_strided(t.shape, (ld, 1))
        return store, view.copy_(t)

    flat = lambda t: torch.empty(t.numel() + offset, device="cuda", dtype=dtype)[offset:].copy_(t.reshape(-1))
    nb = eq.add_adapters_workspace_bytes(tokens, n, k, rank, 3)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    for extra in (0, 1, 8):
        (_, vy), (_, vx), (so, vo) = place(y, n + extra), place(x, k + extra), place(y * 0, n + extra)
        eq.add_adapters(vy, n + extra, vx, k + extra, flat(a), flat(b), index, scale, eq.BF16, tokens, n, k, rank, 3, vo, n + extra, ws, nb, stream)
        assert_same(vo)
        vo.fill_(-77.0)
        assert bool((so == -77.0).all())
        eq.add_adapters(vy, n + extra, vx, k + extra, a, b, index, scale, eq.BF16, tokens, n, k, rank, 3, vy, n + extra, ws, nb, stream)
        assert_same(vy)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("beside", [0, 8])
@pytest.mark.parametrize("tokens,n,k,rank,count", [(9, 33, 72, 16, 3), (3000, 1001, 640, 64, 2), (2500, 541, 1000, 8, 5), (5000, 5, 648, 16, 3),
                                                   (3001, 131, 64, 128, 2), (4000, 190, 777, 16, 2), (20001, 63, 136, 32, 9)])
def test_what_lies_beside_an_output_stays(dtype, beside, tokens, n, k, rank, count):
    """outputs that are columns of a wider tensor, of a width that fills no 16 bytes, apart from y and in its place"""
    y, x, a, b, scale = inputs(tokens, n, k, rank, count, 1, dtype)
    for index in patterns(tokens, count, tokens):
        store, _, view = padded(tokens, n, dtype, beside)
        wide, _, same = padded(tokens, n, dtype, beside)
        same.copy_(y)
        assert ad.add_adapters(same, x, a, b, index, scale, out=view) is view
        check(view, y, x, a, b, index, scale)
        assert torch.equal(ad.add_adapters(same, x, a, b, index, scale, out=same), view)
        assert_beside(store, n), assert_beside(wide, n)


@gpu
def test_offsets_beyond_32_bits():
    dtype, ld = torch.bfloat16, 1 << 26
    y, x, a, b, scale = inputs(70, 96, 64, 16, 5, 1, dtype)
    index = patterns(70, 5, 3)[1]
    want = ad.add_adapters(y, x, a, b, index, scale)
    store = torch.empty(69 * ld + 4096, dtype=dtype, device="cuda")
    fy, fx, fo = (store.as_strided((70, w), (ld, 1), at) for w, at in ((96, 0), (64, 1024), (96, 2048)))
    fy.copy_(y), fx.copy_(x)
    assert torch.equal(ad.add_adapters(fy, fx, a, b, index, scale), want)
    assert torch.equal(ad.add_adapters(fy, fx, a, b, index, scale, out=fo), want)
    # adapters whose last one lies 2^32 elements after the first
    del store, fy, fx, fo
    count = 66000
    big = torch.empty(count, 16, 4096, dtype=dtype, device="cuda")
    xx, bb = normal(3, 4096, 5, dtype), normal(count * 8, 16, 6, dtype).view(count, 8, 16)
    last = normal(16, 4096, 7, dtype, 2.0 ** -6)
    big[-1], big[7] = last, last
    bb[7] = bb[-1]
    yy = normal(3, 8, 8, dtype)
    at = lambda i: torch.full((3,), i, dtype=torch.int32, device="cuda")
    assert torch.equal(ad.add_adapters(yy, xx, big, bb, at(count - 1)), ad.add_adapters(yy, xx, big, bb, at(7)))
    # the same through tiles: the adapters that follow one another end at that one
    xx, yy = normal(3000, 4096, 5, dtype), normal(3000, 8, 8, dtype)
    few = big[-3:]
    index = (torch.arange(3000) % 3).int().cuda()
    want = ad.add_adapters(yy, xx, few.contiguous(), bb[-3:].contiguous(), index)
    assert eq.add_adapters_workspace_bytes(3000, 8, 4096, 16, 3) > 0
    assert torch.equal(ad.add_adapters(yy, xx, few, bb[-3:], index), want)


@gpu
def test_no_tokens_no_adapters_streams_graphs():
    dtype = torch.bfloat16
    y, x, a, b, scale = inputs(100, 96, 64, 16, 5, 1, dtype)
    index = patterns(100, 5, 3)[1]
    assert ad.add_adapters(y[:0], x[:0], a, b, index[:0]).shape == (0, 96)
    assert torch.equal(ad.add_adapters(y, x, a[:0], b[:0], index), y)
    want = ad.add_adapters(y, x, a, b, index, scale)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [ad.add_adapters(y * 1, x, a, b, index, scale) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, want) for t in got)
    many = inputs(3000, 520, 512, 32, 3, 5, dtype)                  # tiles of tokens
    mixed = patterns(3000, 3, 6)[1]
    tiles = ad.add_adapters(*many[:4], mixed, many[4])
    assert torch.equal(ad.add_adapters(many[0], many[1], many[2][:0], many[3][:0], mixed), many[0])
    w = ff.fp4_quantize(normal(96, 64, 9, dtype))
    base = ff.fp4_linear(x, w)
    both = ad.add_adapters(base, x, a, b, index, scale)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ff.fp4_linear(x, w)
        ad.add_adapters(out, x, a, b, index, scale, out=out)
        out2 = ad.add_adapters(*many[:4], mixed, many[4])
    for _ in range(3):
        out.zero_(), out2.zero_()
        graph.replay()
        assert torch.equal(out, both) and torch.equal(out2, tiles)
    ff.check()


@gpu
def test_what_is_refused_on_the_gpu(monkeypatch):
    dtype = torch.bfloat16
    y, x, a, b, scale = inputs(6, 96, 64, 16, 5, 1, dtype)
    index = patterns(6, 5, 3)[0]
    for bad in ((y, x[:5], a, b, index), (y, x, a[:, :, :63], b, index), (y, x, a.half(), b, index), (y, x, a, b[:4], index),
                (y, x, a, b[:, :, :8], index), (y, x, a, b, index.long()), (y, x, a, b, index[:5]), (y, x, a, b, index, scale[:4]),
                (y, x, a, b, index, scale.half()), (y, x, a, b, index, scale, x), (y.float(), x, a, b, index)):
        with pytest.raises(ValueError):
            ad.add_adapters(*bad)
    with pytest.raises(eq.EquarxError):
        ad.add_adapters(y, x, a, b, index, scale, y.as_strided((6, 96), (64, 1)))
    for i in range(4):
        args = [y, x, a, b]
        args[i] = args[i].clone().requires_grad_()
        with pytest.raises(ValueError, match="no_grad"):
            ad.add_adapters(*args, index)
        with torch.no_grad():
            ad.add_adapters(*args, index)
    monkeypatch.setenv("EQUARX_INJECT_LAUNCH_ERROR", "719")
    with pytest.raises(eq.EquarxError) as err:
        ad.add_adapters(y, x, a, b, index)
    assert err.value.status == binding.ERR_CUDA and eq.last_cuda_error() == 719


@gpu
def test_a_wait_of_the_adapters_that_runs_out_is_reported_once(monkeypatch):
    """their waits have a count of their own, which the check reads too; the context stays usable"""
    dtype = torch.bfloat16
    y, x, a, b, scale = inputs(3000, 520, 512, 32, 3, 5, dtype)     # tiles of tokens, whose kernel waits
    index = patterns(3000, 3, 6)[0]
    want = ad.add_adapters(y, x, a, b, index, scale)
    ff.check()
    for names in (["EQUARX_INJECT_TIMEOUT_ADAPTERS"], ["EQUARX_INJECT_TIMEOUT_ADAPTERS", "EQUARX_INJECT_TIMEOUT"]):
        for name in names:
            monkeypatch.setenv(name, "50")                          # 0.2 ms
        with pytest.raises(eq.EquarxError) as err:
            ff.check()
        assert err.value.status == binding.ERR_TIMEOUT
        for name in names:
            monkeypatch.delenv(name)
        ff.check()
    assert torch.equal(ad.add_adapters(y, x, a, b, index, scale), want)
