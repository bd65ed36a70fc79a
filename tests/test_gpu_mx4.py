"""Microscaled 4-bit floating point: quantisation bit for bit, products and 1x1 convolutions against the definition in 64 bits.

Products are of numbers of 2 bits each times powers of two, exact in fp32; only their sums round.  A sum over K values is made of
at most K/32 + 64 additions one after another (the matrix instruction adds up a block of k at a time, wavefronts that share a
sum add their parts), each off by at most a step, 2 E, of the magnitudes summed; bias, residual and activation add 16 E of theirs.
"""
import pytest
import torch

import mx4_reference as R

pytestmark = pytest.mark.gpu
E = R.E24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _same(got, want):
    return torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (7, 64), (1000, 150), (129, 96), (257, 8), (2, 8200), (4096, 256), (33, 2047), (0, 64), (511, 100)])
def test_quantisation_is_exact(rows, cols, dtype):
    from paper_2211_03715_amd import mx4
    g = _gen(rows * 10007 + cols)
    x = (torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-12, 12, (rows, 1), generator=g).float())).to(dtype)
    want = R.quantize(x)
    got = mx4.quantize(x.cuda())
    assert _same(got, want)
    v = R.values(*want, cols)
    for out in (F32, F16, BF16):
        assert torch.equal(mx4.dequantize(*got, cols, dtype=out).cpu().double(), v.to(out).double())


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
def test_every_border_at_every_scale(dtype):
    """Borders between codes, their neighbours in the type on both sides, and the largest value of the block at every exponent."""
    from paper_2211_03715_amd import mx4
    lo, hi = {F32: (-149, 127), F16: (-24, 15), BF16: (-133, 127)}[dtype]
    border = torch.tensor([.25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    rows = []
    for e in range(lo, hi + 1):
        b = torch.ldexp(border.double(), torch.tensor(e - 2)).to(dtype)
        ints = {F32: torch.int32, F16: torch.int16, BF16: torch.int16}[dtype]
        up, down = (b.view(ints) + 1).view(dtype), (b.view(ints) - 1).view(dtype)
        down = torch.where(b == 0, b, down)
        top = torch.ldexp(torch.ones(1, dtype=torch.float64), torch.tensor(e)).to(dtype)
        for part in (b, up, down):
            part = torch.where(part.double().abs() < 2.0 ** (e + 1), part, torch.zeros_like(part))
            rows.append(torch.cat((top, part * (1 - 2 * (torch.arange(15) % 2)).to(dtype), torch.zeros(16, dtype=dtype))))
    x = torch.stack(rows)
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    assert _same(mx4.quantize(x.cuda()), R.quantize(x))


def test_zeros_infinities_and_nans():
    from paper_2211_03715_amd import mx4
    x = torch.randn((6, 70), generator=_gen(1))
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 40] = float("nan")
    x[3, 69] = -float("inf")
    x[4, :32] = -0.0
    x[5, 0] = 3.4e38
    got, want = mx4.quantize(x.cuda()), R.quantize(x)
    assert _same(got, want)
    y = mx4.dequantize(*got, 70).cpu()
    assert torch.equal(torch.isnan(y), torch.isnan(R.values(*want, 70)))
    assert bool(torch.isnan(y[1, :32]).all()) and bool(torch.isfinite(y[1, 32:]).all()) and bool(torch.isnan(y[3, 64:]).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("cols,extra,offset", [(64, 64, 0), (60, 4, 4), (33, 7, 1), (32, 1, 0), (100, 3, 2)])
def test_rows_apart(cols, extra, offset, dtype):
    from paper_2211_03715_amd import mx4
    wide = torch.randn((3, 11, cols + extra + offset), generator=_gen(cols)).to(dtype)
    x = wide[..., offset:offset + cols]
    assert _same(mx4.quantize(wide.cuda()[..., offset:offset + cols]), R.quantize(x))
    with pytest.raises(ValueError):
        mx4.quantize(wide.cuda()[:, ::2, :cols])         # 11 rows give 6: images are no longer evenly spaced
    with pytest.raises(ValueError):
        mx4.quantize(wide.cuda().transpose(0, 2))


def _random_pair(rows, cols, seed):
    return R.quantize(torch.randn((rows, cols), generator=_gen(seed)) * torch.exp2(2 * torch.randn((rows, 1), generator=_gen(seed + 1)).clamp(-2, 2)))


def _cuda(pair):
    return tuple(t.cuda() for t in pair)


def _product(av, bv, bias, res, act, K):
    """The product in 64 bits and what fp32 sums may be off by."""
    v, mag = av @ bv.t(), av.abs() @ bv.abs().t()
    err = 2 * E * (K / 32 + 64) * mag
    for extra in (bias, res):
        if extra is not None:
            v, err = v + extra.double(), err + 16 * E * extra.double().abs()
    return R.act(v, act), 1.1 * err + 16 * E * v.abs()


# M, N, K: one of each, borders of blocks and tiles, one row, few rows, few columns, long sums, more than a tile each way
PRODUCTS = [(1, 1, 1), (1, 1000, 2048), (1, 33, 8192), (2, 16, 32), (3, 17, 65), (16, 64, 512), (17, 129, 100), (31, 31, 31), (33, 40, 96), (64, 256, 256), (65, 257, 160),
            (100, 10, 300), (127, 130, 1000), (128, 128, 2080), (300, 520, 768), (512, 1024, 1024), (1000, 300, 4096), (4, 2000, 4100), (700, 64, 64), (2049, 129, 33), (257, 513, 8200),
            (1024, 768, 256), (48, 4096, 544), (515, 772, 1280),
            # large tiles and smaller ones, from one step of k to many, with whole and broken groups of four blocks
            (1100, 1030, 20), (1100, 1030, 250), (1152, 1024, 384), (1030, 1100, 544), (1025, 1300, 1000), (2900, 3000, 100), (3000, 2817, 33), (2817, 3000, 512), (2900, 2900, 1300)]


@pytest.mark.parametrize("shape", PRODUCTS, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
def test_product(shape, dtype):
    from paper_2211_03715_amd import mx4
    M, N, K = shape
    act = ("none", "relu", "silu")[(M + N) % 3]
    print("[case] product", shape, dtype, act, flush=True)
    a, b = _random_pair(M, K, M + K), _random_pair(N, K, N + 3 * K)
    g = _gen(M + N + K)
    bias = torch.randn(N, generator=g) if M % 2 else None
    res = torch.randn((M, N), generator=g).to(dtype) if N % 2 == 0 else None
    y = torch.full((M, N), float("nan"), device="cuda", dtype=dtype)
    mx4.matmul(_cuda(a), _cuda(b), K, bias=None if bias is None else bias.cuda(), residual=None if res is None else res.cuda(), act=act, dtype=dtype, y=y)
    want, err = _product(R.values(*a, K), R.values(*b, K), bias, res, act, K)
    R.assert_within(y, want, err, dtype, "y")


def test_scales_at_both_ends_and_nan_blocks():
    """Products of scales far apart, sums that overflow to infinity, values that vanish, and a NaN block in one row and one column."""
    from paper_2211_03715_amd import mx4
    K = 96
    a, b = _random_pair(40, K, 1), _random_pair(36, K, 2)
    for i, e in enumerate((0, 1, 60, 200, 250)):
        a[1][i] = e
    for i, e in enumerate((254, 127, 60, 40)):
        b[1][i] = e
    a[1][20, 1] = 255
    b[1][30, 2] = 255
    y = mx4.matmul(_cuda(a), _cuda(b), K).cpu().double()
    want, err = _product(R.values(*a, K), R.values(*b, K), None, None, "none", K)
    # A partial sum may reach the sum of the magnitudes and overflow on the way to a small result: the numbers are those whose
    # magnitudes sum to less than the largest float, 2^128.
    mag = R.values(*a, K).abs() @ R.values(*b, K).abs().t()
    fine = ~torch.isnan(want) & (mag < 2.0 ** 127)
    assert torch.equal(torch.isnan(y)[fine | torch.isnan(want)], torch.isnan(want)[fine | torch.isnan(want)])
    # below 2^-126 the sums are multiples of 2^-149, and the products of two scales below 2^-149 are zeros: 2^-126 covers them
    assert bool(((y - want).abs()[fine] <= err[fine] + 2.0 ** -126).all())
    huge = want.abs() >= 2.0 ** 129
    assert not bool(torch.isfinite(y[huge & ~torch.isnan(want)]).any())
    assert bool(torch.isnan(y[20]).all()) and bool(torch.isnan(y[:, 30]).all()) and bool(torch.isfinite(y[19, 1:30]).all())   # column 0's scale is 2^127


# batch, H, W, C, N, stride, extra pixel pitch
CONVS = [(1, 1, 1, 2048, 1000, 1, 0), (1, 1, 1, 33, 5, 1, 0), (1, 7, 7, 512, 128, 1, 0), (2, 9, 7, 100, 150, 2, 0), (3, 5, 5, 64, 64, 3, 0), (2, 8, 8, 96, 256, 2, 32), (1, 3, 2, 30, 40, 1, 3),
         (4, 28, 28, 128, 512, 1, 0), (2, 56, 56, 64, 48, 1, 0), (16, 1, 1, 1024, 333, 1, 0), (1, 4, 4, 4096, 64, 1, 0), (2, 15, 15, 260, 1030, 2, 4), (40, 1, 1, 320, 96, 1, 0), (8, 30, 30, 32, 16, 1, 0)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("shape", CONVS, ids=lambda s: "x".join(map(str, s)))
def test_convolution(shape, dtype):
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    batch, H, W, C, N, stride, extra = shape
    act = ("none", "relu", "silu")[(H + C + N) % 3]
    print("[case] conv", shape, dtype, act, flush=True)
    g = _gen(C * 7 + N)
    wide = torch.randn((batch, H, W, C + extra), generator=g).to(dtype)
    x = wide[..., :C]
    Wt = torch.randn((C, N, 1, 1), generator=g) * C ** -0.5
    bias = torch.randn(N, generator=g)
    conv = mx4.MX4Conv2d(Layer(batch, C, N, H, W, 1, 1, 1, stride, 0), dtype=dtype, x_pitch=C + extra)
    conv.pack(Wt.cuda())
    res = torch.randn(conv.out_shape(), generator=g).to(dtype) if N % 2 == 0 else None
    y = torch.full(conv.out_shape(), float("nan"), device="cuda", dtype=dtype)
    extras = {"bias": bias.cuda(), "residual": None if res is None else res.cuda(), "act": act}
    conv(wide.cuda()[..., :C], y, **extras)
    wv = R.values(*R.quantize(Wt.reshape(C, N).t()), C)
    xs = x[:, ::stride, ::stride]
    xv = R.values(*R.quantize(xs), C)
    want, err = _product(xv.reshape(-1, C), wv, bias, None if res is None else res.reshape(-1, N), act, C)
    R.assert_within(y.reshape(-1, N), want, err, dtype, "y")
    # the same from x in 4 bits: what is quantised on the way is what quantize() gives, but sums may be split otherwise
    z = conv(mx4.quantize(x.contiguous().cuda()), **extras)
    R.assert_within(z.reshape(-1, N), want, err, dtype, "y from 4 bits")


def test_convolution_of_what_is_no_number():
    """A NaN or an infinity makes the outputs of its pixel NaN, and no others."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    for batch, H in ((1, 3), (2, 20)):
        conv = mx4.MX4Conv2d(Layer(batch, 64, 48, H, H, 1, 1, 1, 1, 0))
        conv.pack(torch.randn((64, 48), generator=_gen(1)).cuda())
        x = torch.randn((batch, H, H, 64), generator=_gen(2))
        x[0, 1, 1, 40] = float("nan")
        x[0, 2, 1, 3] = float("inf")
        for act in ("none", "relu"):
            y = conv(x.cuda(), act=act).cpu()
            nan = torch.isnan(y)
            assert bool(nan[0, 1, 1].all()) and bool(nan[0, 2, 1].all()) and int(nan.sum()) == 2 * 48


def test_repacked_weights_and_the_same_bits_again():
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    conv = mx4.MX4Conv2d(Layer(2, 128, 96, 14, 14, 1, 1, 1, 1, 0))
    x = torch.randn((2, 14, 14, 128), generator=_gen(3)).cuda()
    with pytest.raises(Exception):
        conv(x)                                        # no weights yet
    ys = []
    for seed in (4, 5, 4):
        conv.pack(torch.randn((128, 96, 1, 1), generator=_gen(seed)).cuda())   # the tensor may go at once
        ys.append(conv(x))
        assert torch.equal(ys[-1], conv(x))
    assert torch.equal(ys[0], ys[2]) and not torch.equal(ys[0], ys[1])


def test_norm_and_convolution_together_on_a_stream_and_in_a_graph():
    """The end of a bottleneck block: norm + activation in 4 bits, 1x1 convolution, bias, shortcut; eagerly, on a stream of its
    own with the weights packed on another, and as a graph replayed on changing inputs with eager calls in between."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.norm import GroupNorm
    from paper_2211_03715_amd.workloads import Layer
    B, H, C, N = 2, 14, 64, 256
    g = _gen(7)
    xs = [torch.randn((B, H, H, C), generator=g) for _ in range(3)]
    gamma, beta, bias = (torch.randn(n, generator=g) for n in (C, C, N))
    Wt, res = torch.randn((C, N, 1, 1), generator=g) * C ** -0.5, torch.randn((B, H, H, N), generator=g)
    gn = GroupNorm(B, H, H, C, 8, act="relu")
    conv = mx4.MX4Conv2d(Layer(B, C, N, H, H, 1, 1, 1, 1, 0))
    conv.pack(Wt.cuda(), stream=torch.cuda.Stream())
    gd, bd, biasd, resd = gamma.cuda(), beta.cuda(), bias.cuda(), res.cuda()

    def block(x, stream=None):
        return conv(gn.quantized(x, gd, bd, stream=stream), bias=biasd, residual=resd, act="relu", stream=stream)

    wv = R.values(*R.quantize(Wt.reshape(C, N).t()), C)
    want = []
    for x in xs:
        y = block(x.cuda())
        normed = gn(x.cuda(), gd, bd).cpu()            # the values that were quantised, in fp32
        v, err = _product(R.values(*R.quantize(normed), C).reshape(-1, C), wv, bias, res.reshape(-1, N), "relu", C)
        R.assert_within(y.reshape(-1, N), v, err, F32, "block")
        want.append(y)
    side = torch.cuda.Stream()
    x = xs[2].cuda()
    torch.cuda.synchronize()
    y = block(x, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(y, want[2])
    static = torch.zeros_like(x)
    block(static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(static)
    for i in (1, 0, 2, 1):
        static.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), i
        assert torch.equal(block(xs[(i + 1) % 3].cuda()), want[(i + 1) % 3])
        torch.cuda.synchronize()


def test_bound_launchers():
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.norm import GroupNorm
    from paper_2211_03715_amd.workloads import Layer
    x = torch.randn((1, 5, 6, 48), generator=_gen(9)).cuda()
    gn, conv = GroupNorm(1, 5, 6, 48, 4, act="silu"), mx4.MX4Conv2d(Layer(1, 48, 40, 5, 6, 1, 1, 1, 1, 0))
    conv.pack(torch.randn((48, 40), generator=_gen(8)).cuda())
    y, z, q = torch.empty_like(x), torch.empty(conv.out_shape(), device="cuda"), gn.new_quantized()
    gn.bind(x, y)()
    assert torch.equal(y, gn(x))
    conv.bind(y, z)()
    assert torch.equal(z, conv(y))
    gn.bind_quantized(x, q)()
    conv.bind(q, z)()
    assert torch.equal(z, conv(gn.quantized(x)))


def test_refusals_of_the_layer():
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    conv = mx4.MX4Conv2d(Layer(2, 64, 32, 4, 4, 1, 1, 1, 1, 0))
    for bad in (torch.zeros(32, 64, 1, 1), torch.zeros(64, 32).cuda().half(), torch.zeros(64, 32), torch.zeros(32, 64).cuda().t()):
        with pytest.raises(ValueError):
            conv.pack(bad)
    conv.pack(torch.zeros(64, 32).cuda())
    x = torch.zeros((2, 4, 4, 64), device="cuda")
    for bad in (x.half(), x[:1], x.cpu(), torch.zeros((2, 4, 4, 96), device="cuda")[..., :64], mx4.quantize(x[:1])):
        with pytest.raises(ValueError):
            conv(bad)
    for kw in (dict(bias=torch.zeros(31).cuda()), dict(bias=torch.zeros(32)), dict(residual=torch.zeros((2, 4, 4, 32)).cuda().half()), dict(act="tanh"), dict(y=torch.zeros(2, 4, 4, 32))):
        with pytest.raises(ValueError):
            conv(x, **kw)
    codes, scales = mx4.quantize(x)
    for bad in ((codes, scales, 65), (codes, scales[:1], 64), (codes[..., :16], scales, 64), (codes.cpu(), scales, 64), (codes, scales, 0)):
        with pytest.raises(ValueError):
            mx4.dequantize(*bad)
    a = mx4.quantize(x.reshape(-1, 64))
    with pytest.raises(ValueError):
        mx4.matmul(a, mx4.quantize(x), 64)
    with pytest.raises(ValueError):
        mx4.matmul(a, a, 96)
    with pytest.raises(ValueError):
        mx4.matmul(a, a, 64, dtype=torch.float64)
    assert mx4.matmul(tuple(t[:0].contiguous() for t in a), a, 64).shape == (0, 32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,pitch", [(7, 64, 96), (5, 33, 40), (300, 24, 25), (1, 5, 9)])
def test_values_written_apart(rows, cols, pitch, dtype):
    """tdc_mx4_dequantize with a pitch: what lies between the rows stays as it was."""
    from paper_2211_03715_amd import binding as B
    x = torch.randn((rows, cols), generator=_gen(rows)).to(dtype)
    codes, scales = R.quantize(x)
    wide = torch.full((rows, pitch), 7.0, dtype=dtype, device="cuda")
    c, s = codes.cuda(), scales.cuda()
    code = {F32: 0, BF16: 2}[dtype]
    assert B.load().tdc_mx4_dequantize(torch.cuda.current_stream().cuda_stream, c.data_ptr(), s.data_ptr(), rows, cols, wide.data_ptr(), code, pitch) == B.TDC_OK
    wide = wide.cpu()
    assert torch.equal(wide[:, :cols].double(), R.values(codes, scales, cols).to(dtype).double()) and bool((wide[:, cols:] == 7).all())
