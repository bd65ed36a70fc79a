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
