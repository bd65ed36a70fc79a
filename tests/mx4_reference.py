"""The operators of tdc_norm.h and tdc_mx4.h from their definitions, in 64 bits on the CPU (torch, float64)."""
import torch

E24 = 2.0 ** -24                                   # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step of each type
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}                # half of fp16's smallest step


def act(v, name):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    return v * torch.sigmoid(v) if name == "silu" else v


def group_norm(x, groups, eps, gamma=None, beta=None, residual=None):
    """(pre, xhat, mean [B][G], rstd) of x [B][H][W][C], all float64."""
    B, H, W, C = x.shape
    v = x.double().reshape(B, H * W, groups, C // groups)
    mean = v.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + eps)
    xhat = ((v - mean) * rstd).reshape(x.shape)
    pre = xhat if gamma is None else xhat * gamma.double()
    pre = pre if beta is None else pre + beta.double()
    pre = pre if residual is None else pre + residual.double()
    return pre, xhat, mean.reshape(B, groups), rstd.reshape(B, groups)


VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def quantize(x):
    """Codes [..., 16 nb] and scales [..., nb] (uint8) of x [..., C]: nearest value by search, ties to the even code."""
    C = x.shape[-1]
    nb = -(-C // 32)
    v = torch.zeros(x.shape[:-1] + (nb * 32,), dtype=torch.float64)
    v[..., :C] = x.double()
    v = v.reshape(-1, 32)
    bad = ~torch.isfinite(v).all(1, keepdim=True)
    v = torch.where(bad, torch.zeros_like(v), v)
    top = v.abs().amax(1, keepdim=True)
    e = torch.clamp(torch.frexp(top).exponent.double() - 1 - 2, -127, 127)
    e = torch.where(top > 0, e, torch.full_like(e, -127.0))
    a = (v.abs() * torch.pow(2.0, -e)).clamp(max=6)
    gap = (a[..., None] - VALUES).abs()
    near = gap == gap.amin(-1, keepdim=True)           # one code, or two next to each other at a tie
    code = torch.arange(8) + 8 * (torch.arange(8) % 2)  # even codes first
    code = torch.where(near, code, torch.full_like(code, 99)).amin(-1) % 8
    code = code + 8 * torch.signbit(v).long()
    code = torch.where(bad, torch.zeros_like(code), code)
    packed = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8)
    scale = torch.where(bad, torch.full_like(e, 255.0), e + 127).to(torch.uint8)
    return packed.reshape(x.shape[:-1] + (nb * 16,)), scale.reshape(x.shape[:-1] + (nb,))


def values(codes, scales, C):
    """float64 values [..., C]."""
    n = torch.stack((codes & 15, codes >> 4), -1).reshape(scales.shape + (32,)).long()
    v = VALUES[n % 8] * (1 - 2 * (n // 8).double())
    s = torch.where(scales == 255, torch.full(scales.shape, float("nan"), dtype=torch.float64), torch.pow(2.0, scales.double() - 127))
    return (v * s[..., None]).reshape(scales.shape[:-1] + (scales.shape[-1] * 32,))[..., :C]


def assert_within(got, want, bound, dtype, what=""):
    """|got - want| <= bound (fp32 arithmetic) + half a step of dtype, where want is a number; the same NaNs and infinities elsewhere."""
    got, want = got.detach().cpu().double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaNs differ" % what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), "%s: infinities differ" % what
    bound = torch.as_tensor(bound, dtype=torch.float64).expand(want.shape)
    limit = bound + (want.abs() + bound) * HALF[dtype] + TINY[dtype]
    over = ((got - want).abs() - limit)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, "%s: off by %.3g where %.3g is allowed (%d of %d)" % (
        what, float((got - want).abs()[fine][over.argmax()]), float(limit[fine][over.argmax()]), int((over > 0).sum()), over.numel())
