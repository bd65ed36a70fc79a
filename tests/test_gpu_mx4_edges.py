"""4-bit quantisation, products and convolutions at the ends of what they take, and through every kernel that a call can choose.

Tolerances as in test_gpu_mx4.py, whose bound of a product's sums is used."""
import pytest
import torch

import mx4_reference as R
from test_gpu_mx4 import _product, _random_pair

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture
def room():
    """Sizes that need tens of GB: what earlier tests left in the allocator's pool goes first, and what these take goes behind them."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_as_many_blocks_as_a_call_takes(room):
    """2^31 - 128 rows of one value: its scale byte is its exponent's less 2, and what comes back has its two leading bits."""
    from paper_2211_03715_amd import mx4
    n = 2 ** 31 - 128
    x = torch.empty((n, 1), device="cuda", dtype=BF16).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    codes, scales = mx4.quantize(x)
    y = mx4.dequantize(codes, scales, 1, dtype=BF16)
    for a, c, s, b in zip(*(t.reshape(n, -1).split(1 << 26) for t in (x, codes, scales, y))):
        v = a.float()
        e = torch.frexp(v).exponent - 1
        want = torch.where(v == 0, torch.zeros_like(e), e + 125)
        assert torch.equal(s.int(), want.int())
        # 4 to 8 in units of the scale: 4 up to 5, a tie that goes to 4; 6 from there on
        unit = torch.ldexp(torch.ones_like(v), e - 2)
        code = torch.where(v == 0, 0, torch.where(v.abs() > 5 * unit, 7, 6)) + 8 * torch.signbit(v)
        assert torch.equal(c[:, 0].int(), code[:, 0].int()) and not bool(c[:, 1:].any())
        assert torch.equal(b.float(), torch.copysign(torch.where(v == 0, torch.zeros_like(v), torch.where(v.abs() > 5 * unit, 6 * unit, 4 * unit)), v))


def test_a_convolution_of_as_many_pixels_as_a_plan_takes(room):
    """2^29 - 32 pixels, one channel in and out: products of two numbers of two bits are exact in bf16."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    n = 2 ** 29 - 32
    x = torch.empty((1, 1, n, 1), device="cuda", dtype=BF16).normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    w = torch.full((1, 1), 0.75, device="cuda")
    conv = mx4.MX4Conv2d(Layer(1, 1, 1, 1, n, 1, 1, 1, 1, 0), dtype=BF16)
    conv.pack(w)
    y, v = conv(x), mx4.dequantize(*mx4.quantize(x), 1, dtype=BF16)
    for a, b in zip(y.reshape(-1).split(1 << 26), v.reshape(-1).split(1 << 26)):
        assert torch.equal(a.float(), 0.75 * b.float())


def test_every_fifth_of_2_31_pixels(room):
    """The largest image, one channel in and out; what is read lies up to 2^31 - 2 pixels in."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    n = 2 ** 31 - 1
    x = torch.empty((1, n, 1, 1), device="cuda", dtype=BF16).normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    conv = mx4.MX4Conv2d(Layer(1, 1, 1, n, 1, 1, 1, 1, 5, 0), dtype=BF16)
    conv.pack(torch.full((1, 1), 0.75, device="cuda"))
    y, q = conv(x), mx4.quantize(x[:, ::5].contiguous())
    v = mx4.dequantize(*q, 1, dtype=BF16)
    assert y.shape == v.shape
    for a, b in zip(y.reshape(-1).split(1 << 26), v.reshape(-1).split(1 << 26)):
        assert torch.equal(a.float(), 0.75 * b.float())


def test_a_convolution_with_more_than_2_33_outputs(room):
    """64 images of 224 x 224, 64 channels to 4096: 2^33.6 outputs of 16 bits.  Some pixels of each image are looked at."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    B, H, C, N = 64, 224, 64, 4096
    g = torch.Generator().manual_seed(3)
    x = torch.empty((B, H, H, C), device="cuda", dtype=BF16).normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    W = torch.randn((C, N), generator=g) * C ** -0.5
    conv = mx4.MX4Conv2d(Layer(B, C, N, H, H, 1, 1, 1, 1, 0), dtype=BF16)
    conv.pack(W.cuda())
    y = conv(x).reshape(-1, N)
    some = torch.cat((torch.randint(0, B * H * H, (40,), generator=g), torch.tensor([0, B * H * H - 1])))
    xv, wv = R.values(*R.quantize(x.reshape(-1, C)[some.cuda()].cpu()), C), R.values(*R.quantize(W.t()), C)
    want, err = _product(xv, wv, None, None, "none", C)
    R.assert_within(y[some.cuda()], want, err, BF16, "y")


def test_a_product_with_2_33_outputs(room):
    from paper_2211_03715_amd import mx4
    M, N, K = 65536, 131072, 64
    a, b = _random_pair(M, K, 4), _random_pair(N, K, 5)
    y = mx4.matmul(tuple(t.cuda() for t in a), tuple(t.cuda() for t in b), K, dtype=BF16)
    some = torch.tensor([0, 1, 255, 256, 32767, 32768, 50001, M - 1])
    want, err = _product(R.values(a[0][some], a[1][some], K), R.values(*b, K), None, None, "none", K)
    R.assert_within(y[some.cuda()], want, err, BF16, "y")


# ---- every kernel that a convolution can choose

def _values(q, C):
    """R.values on the GPU."""
    codes, scales = q
    n = torch.stack((codes & 15, codes >> 4), -1).reshape(scales.shape + (32,)).long()
    v = R.VALUES.to(codes.device)[n % 8] * (1 - 2 * (n // 8).double()) * torch.pow(2.0, scales.double() - 127)[..., None]
    return v.reshape(scales.shape[:-1] + (-1,))[..., :C]


def _way(batch, H, W, C, N, stride):
    """As tdc_mx4_internal.h chooses: products in large tiles; a workgroup to 32 rows and 64 columns, eight wavefronts along k; or a
    workgroup to 32 rows, its wavefronts at 64 columns each."""
    rows = batch * ((H - 1) // stride + 1) * ((W - 1) // stride + 1)
    if rows >= 4096 and N >= 1024 and C >= 1024:
        return "large"
    return "few" if -(-rows // 32) * -(-N // 64) <= 512 else "many"


# batch, H, W, C, N, stride, extra pixel pitch: ragged columns, pixels in whole pieces and not, every second or third pixel, gaps between
# pixels, k beyond what LDS holds at a time (8192)
WAYS = [("many", (8, 60, 60, 100, 150, 1, 0)), ("many", (8, 61, 59, 104, 151, 2, 0)), ("many", (2, 100, 100, 264, 330, 1, 8)), ("many", (1, 130, 131, 33, 65, 1, 3)), ("many", (8, 90, 88, 40, 1000, 3, 1)),
        ("many", (32, 28, 28, 128, 512, 1, 0)), ("many", (1, 73, 76, 8232, 190, 1, 0)), ("many", (1, 73, 76, 8225, 190, 1, 0)),
        ("large", (16, 17, 19, 1056, 1040, 1, 0)), ("large", (8, 47, 45, 1030, 1028, 2, 2)), ("large", (4, 33, 33, 1024, 1041, 1, 0)), ("large", (5, 30, 29, 2048, 1024, 1, 8)),
        ("few", (1, 4, 4, 9000, 64, 1, 0)), ("few", (1, 9, 9, 2056, 70, 2, 8)), ("few", (5, 9, 9, 65, 33, 1, 0))]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("way,shape", WAYS, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else s)
def test_every_way_of_a_convolution(way, shape, dtype):
    """Against the definition in 64 bits on the blocks that quantize() gives, which test_gpu_mx4.py compares bit for bit."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    batch, H, W, C, N, stride, extra = shape
    assert _way(*shape[:6]) == way
    act = ("none", "relu", "silu")[(H + C + N) % 3]
    print("[case] conv", way, shape, dtype, act, flush=True)
    g = torch.Generator(device="cuda").manual_seed(C * 7 + N)
    randn = lambda *s: torch.randn(s, device="cuda", generator=g)
    wide = randn(batch, H, W, C + extra).to(dtype)
    x, Wt, bias = wide[..., :C], randn(C, N) * C ** -0.5, randn(N)
    conv = mx4.MX4Conv2d(Layer(batch, C, N, H, W, 1, 1, 1, stride, 0), dtype=dtype, x_pitch=C + extra)
    conv.pack(Wt)
    out = conv.out_shape()
    extras = {"bias": bias, "residual": randn(*out).to(dtype) if (N + H) % 2 else None, "act": act}
    q = mx4.quantize(x)
    y, z = conv(x, torch.full(out, float("nan"), device="cuda", dtype=dtype), **extras), conv(q, torch.full(out, float("nan"), device="cuda", dtype=dtype), **extras)
    xv = _values(tuple(t[:, ::stride, ::stride].contiguous() for t in q), C).reshape(-1, C)
    wv = _values(mx4.quantize(Wt.t().contiguous()), C)
    res = None if extras["residual"] is None else extras["residual"].reshape(-1, N)
    want, err = _product(xv, wv, bias, res, act, C)
    for got in (y, z):
        R.assert_within(got.reshape(-1, N), want.cpu(), err.cpu(), dtype, "y")
    assert torch.equal(conv(x, **extras), y)


@pytest.mark.parametrize("way,shape", [("many", (2, 100, 100, 96, 200)), ("large", (4, 33, 33, 1024, 1040)), ("few", (2, 5, 5, 96, 200))], ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else s)
def test_what_is_no_number_stays_in_its_pixel(way, shape):
    """An infinity or a NaN makes its pixel's outputs NaN whichever kernel runs, a pixel of zeros gives the bias."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    B, H, W, C, N = shape
    assert _way(*shape, 1) == way
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((B, H, W, C), device="cuda", generator=g)
    bias = torch.randn(N, device="cuda", generator=g)
    conv = mx4.MX4Conv2d(Layer(B, C, N, H, W, 1, 1, 1, 1, 0))
    conv.pack(torch.randn((C, N), device="cuda", generator=g))
    good = conv(x, bias=bias)
    x[0, 1, 2, C - 1], x[1, 3, 0, 5], x[1, 4, 4], x[0, 4, 3, 40] = float("inf"), -float("inf"), 0, float("nan")
    for got in (conv(x, bias=bias), conv(mx4.quantize(x), bias=bias)):
        nan = torch.isnan(got)
        assert all(bool(nan[at].all()) for at in ((0, 1, 2), (1, 3, 0), (0, 4, 3))) and int(nan.sum()) == 3 * N
        assert torch.equal(got[1, 4, 4], bias)
        nan[1, 4, 4] = True
        assert torch.equal(got[~nan], good[~nan])          # the same products in the same order


def test_the_binding_alone():
    """Every function of the binding, on plans and tensors without the layers, gives what the layers give."""
    from paper_2211_03715_amd import binding as B
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.norm import GroupNorm
    from paper_2211_03715_amd.workloads import Layer
    g = torch.Generator(device="cuda").manual_seed(11)
    randn = lambda *s: torch.randn(s, device="cuda", generator=g)
    n, H, C, N, G = 2, 9, 72, 40, 6
    x, dy, res, gamma, beta, W, bias = randn(n, H, H, C), randn(n, H, H, C), randn(n, H, H, C), randn(C), randn(C), randn(C, N), randn(N)
    gn, conv = GroupNorm(n, H, H, C, G, act="silu"), mx4.MX4Conv2d(Layer(n, C, N, H, H, 1, 1, 1, 1, 0))
    conv.pack(W)
    stats = gn.new_stats()
    want = [gn(x, gamma, beta, residual=res, stats=stats), *gn.quantized(x, gamma, beta, residual=res)] + list(gn.backward(x, dy, stats, gamma, beta, residual=res))
    norm = B.tdc_norm_plan_create(B.tdc_norm_shape(n, H, H, C, G, B.F32, B.ACT_SILU, 1e-5))
    assert B.tdc_norm_plan_workspace_bytes(norm) > 0
    assert B.tdc_norm_plan_kernel_count(norm) == gn.kernel_count() and B.tdc_norm_plan_mx4_kernel_count(norm) == gn.kernel_count(quantized=True)
    y, (codes, scales), (mean, rstd) = torch.empty_like(x), gn.new_quantized(), gn.new_stats()
    dx, dres, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    B.tdc_group_norm(norm, x, gamma, beta, y, B.make_norm_args(residual=res, mean=mean, rstd=rstd))
    B.tdc_group_norm_mx4(norm, x, gamma, beta, codes, scales, B.make_norm_args(residual=res))
    B.tdc_group_norm_backward(norm, x, dy, mean, rstd, gamma, beta, dx, dgamma, dbeta, B.make_norm_grad_args(residual=res, dresidual=dres))
    assert all(torch.equal(a, b) for a, b in zip((y, codes, scales, dx, dgamma, dbeta, dres), want))
    B.tdc_norm_plan_destroy(norm)

    rows = x.reshape(-1, C)
    q, w4 = mx4.quantize(rows), mx4.quantize(W.t().contiguous())
    a, b, back, z = torch.empty_like(q[0]), torch.empty_like(q[1]), torch.empty_like(rows), torch.empty((rows.shape[0], N), device="cuda")
    B.tdc_mx4_quantize(rows, B.F32, rows.shape[0], C, a, b)
    B.tdc_mx4_dequantize(a, b, rows.shape[0], C, back, B.F32)
    B.tdc_mx4_matmul(a, b, *w4, rows.shape[0], N, C, z, B.F32, B.make_mx4_epilogue(bias=bias, act=B.ACT_RELU))
    assert torch.equal(a, q[0]) and torch.equal(b, q[1]) and torch.equal(back, mx4.dequantize(*q, C)) and torch.equal(z, mx4.matmul(q, w4, C, bias=bias, act="relu"))
    plan = B.tdc_mx4_plan_create(B.tdc_mx4_shape(n, H, H, C, N, 1, B.F32, 0))
    assert B.tdc_mx4_plan_workspace_bytes(plan) > 0 and B.tdc_mx4_plan_kernel_count(plan) == conv.kernel_count()
    B.tdc_mx4_plan_pack(plan, W)
    c, d = (torch.empty(conv.out_shape(), device="cuda") for _ in range(2))
    B.tdc_conv_mx4(plan, x, c, B.make_mx4_epilogue(bias=bias))
    B.tdc_conv_mx4_quantized(plan, a, b, d)
    assert torch.equal(c, conv(x, bias=bias)) and torch.equal(d, conv(tuple(t.reshape(n, H, H, -1) for t in q)))
    B.tdc_mx4_plan_destroy(plan)
