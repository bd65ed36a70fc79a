"""Group norm through every way that its work is cut up, which the host's choice is asked for beside each case: slices of an image in
256, 512 or 1024 threads, pieces of one channel to 16 bytes, groups of whole pieces or not, ordinary and streaming stores; chunks
of images with or without a launch that combines them, pixels of more pieces than a workgroup has threads, several images to a
workgroup of the backward pass; and each of them written in 4 bits.

Bounds as in test_gpu_norm.py: 64 levels of merging forward and 256 additions backward are not passed by any case here."""
import pytest
import torch

import mx4_reference as R
import norm_choice
from test_gpu_norm import EPS, _inputs, _layer

pytestmark = pytest.mark.gpu
E = R.E24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SIZE = {F32: 4, F16: 2, BF16: 2}


def _vec(C, dtype, most=8):
    v = min(16 // SIZE[dtype], most)
    while C % v:
        v //= 2
    return v


def _forward_path(shape, dtype, mx4=False):
    """(threads or 0, channels to an access, pieces held, streaming stores, whole pieces)."""
    C, G, V = shape[3], shape[4], _vec(shape[3], dtype)
    if mx4 and (C % 32 or V * SIZE[dtype] != 16):
        return (0, V, 0, 0, False)
    s = norm_choice.slices(shape, SIZE[dtype], V, multiple=32 if mx4 else 1)
    return (s["threads"], V, s["held"], s["streams"], C // G % V == 0)


def _backward_path(shape, dtype):
    V = _vec(shape[3], dtype, 4)
    return norm_choice.slices(shape, SIZE[dtype], V, backward=True)["held"], V


def _spread(s, C):
    B, G = s.shape
    return s.reshape(B, 1, 1, G, 1).expand(B, 1, 1, G, C // G).reshape(B, 1, 1, C)


def _forward_want(x, G, act, gamma, beta, res):
    """y in 64 bits, the statistics, and what fp32 may do to y."""
    pre, xhat, mean, rstd = R.group_norm(x, G, EPS, gamma, beta, res)
    B, H, W, C = x.shape
    top = x.double().reshape(B, H * W, G, C // G).abs().amax((1, 3))
    terms = (xhat * gamma).abs() + beta.double().abs() + (0 if res is None else res.double().abs())
    return R.act(pre, act), mean, rstd, 1.1 * E * (48 * terms + 64 * _spread(top * rstd, C) * gamma.double().abs())


def _assert_quantized(q, want, bound):
    """Each block's scale is that of a largest value within the bounds, each value as near to a code as any, within twice the bound."""
    codes, scales = q
    C = want.shape[-1]
    pad = lambda t: torch.nn.functional.pad(t, (0, -C % 32)).reshape(*t.shape[:-1], -1, 32)
    y, err = pad(want), pad(bound)
    top, off = y.abs().amax(-1), err.amax(-1)
    scale = lambda a: torch.where(a > 0, (torch.frexp(a).exponent - 3).clamp(-127, 127) + 127, torch.zeros_like(a).int())
    s = scales.int()
    assert bool(((s >= scale((top - off).clamp(min=0))) & (s <= scale(top + off))).all())
    table = R.VALUES.to(codes.device)
    unit = torch.pow(2.0, s.double() - 127)[..., None]
    n = torch.stack((codes & 15, codes >> 4), -1).reshape(y.shape).long()
    got = table[n % 8] * (1 - 2 * (n // 8).double()) * unit
    near = torch.full_like(y, float("inf"))
    for v in R.VALUES.tolist():
        near = torch.minimum(near, (y.abs() - v * unit).abs())
    assert bool(((got - y).abs() <= near + 2 * err).all())
    assert bool((got[..., -1, (C - 1) % 32 + 1:] == 0).all())


# B, H, W, C, groups and the type's bytes: the least sizes that take each way forward, as `_forward_path` says
FORWARD = [
    # 1024 threads
    (110, 1, 491, 330, 30, 2), (120, 1, 2370, 60, 30, 2), (72, 1, 3691, 64, 16, 2), (33, 1, 2119, 240, 30, 2), (78, 1, 720, 150, 30, 4), (94, 1, 1695, 54, 9, 4),
    (67, 1, 2118, 60, 30, 4), (87, 1, 3021, 32, 8, 4), (32, 56, 56, 256, 32, 4),
    # streaming stores from slices, from chunks
    (32, 28, 28, 512, 32, 2), (32, 28, 28, 512, 32, 4), (8, 28, 28, 480, 40, 4), (8, 28, 28, 480, 48, 2), (2, 100, 100, 256, 2, 4), (2, 100, 100, 264, 3, 2),
    # chunks, pixels of more pieces than threads: whole and not, with and without a launch between; as many groups as channels
    (3, 1, 3, 8191, 1, 4), (3, 1, 3, 8191, 1, 2), (2, 3, 5, 8184, 8, 4), (2, 3, 5, 8184, 8, 2), (2, 2, 2, 8188, 1, 4), (2, 9, 9, 8192, 1, 4), (2, 9, 9, 8192, 2, 2), (1, 1, 4200, 8192, 8192, 2),
    # 4 bits, 16 bits: slices and chunks over lanes, blocks by themselves
    (8, 28, 28, 128, 32, 2), (1, 56, 56, 64, 32, 2), (32, 56, 56, 64, 32, 2), (2, 9, 9, 40, 5, 2), (2, 7, 7, 512, 32, 2), (1, 40, 40, 96, 32, 2), (5, 6, 7, 1024, 64, 2),
]


def _typed(cases):
    name = {F32: "fp32", F16: "fp16", BF16: "bf16"}
    return [pytest.param(c, t, id="x".join(map(str, c[:5])) + "-" + name[t]) for c in cases for t in ((F32,) if c[5] == 4 else (F16, BF16))]


def test_the_cases_take_every_way_forward():
    paths = [_forward_path(c[:5], F32 if c[5] == 4 else BF16) for c in FORWARD]
    assert {(p[0], p[1], p[4]) for p in paths if p[0] == 1024} == {(1024, 2, False), (1024, 4, False), (1024, 8, False), (1024, 8, True), (1024, 2, True), (1024, 4, True)}
    assert any(p[0] == 512 and p[3] for p in paths) and any(p[0] == 0 and p[3] for p in paths)
    four = [_forward_path(c[:5], F32 if c[5] == 4 else BF16, mx4=True) for c in FORWARD]
    assert {p[0] for p in four if p[1] == 8 and p[2]} >= {256, 512}


@pytest.mark.parametrize("case,dtype", _typed(FORWARD))
def test_forward(case, dtype):
    shape = case[:5]
    B, H, W, C, G = shape
    act = ("none", "relu", "silu")[(B + C + H) % 3]
    print("[case] norm", shape, dtype, act, _forward_path(shape, dtype), _forward_path(shape, dtype, True), flush=True)
    x, gamma, beta, res, _ = _inputs(B, H, W, C, dtype, residual=(W + G) % 2 == 1, seed=5)
    x, gamma, beta, res = x.cuda(), gamma.cuda(), beta.cuda(), None if res is None else res.cuda()
    gn = _layer(B, H, W, C, G, act, dtype)
    stats, more = gn.new_stats(), gn.new_stats()
    y = gn(x, gamma, beta, residual=res, stats=stats, y=torch.full_like(x, float("nan")))
    want, mean, rstd, bound = _forward_want(x, G, act, gamma, beta, res)
    R.assert_within(y, want.cpu(), bound.cpu(), dtype, "y")
    q = gn.new_quantized()
    q[0].fill_(0xff), q[1].fill_(0xff)
    assert gn.quantized(x, gamma, beta, residual=res, out=q, stats=more) is q
    _assert_quantized(q, want, bound)
    top = x.double().reshape(B, H * W, G, C // G).abs().amax((1, 3)).cpu()
    for got in (stats, more):
        R.assert_within(got[0], mean.cpu(), 64 * E * top, F32, "mean")
        R.assert_within(got[1], rstd.cpu(), 64 * E * rstd.cpu(), F32, "rstd")


# ways backward: many images in chunks, so that a workgroup takes several; the same with pixels of more pieces than threads, whose
# channels' sums go through memory; slices of every width of piece
BACKWARD = [
    (78, 1, 15097, 1, 1, 2), (7, 1, 13890, 81, 9, 2), (126, 1, 8497, 2, 2, 2), (7, 1, 1489, 690, 30, 2), (87, 1, 10762, 4, 2, 2), (3, 1, 6125, 416, 32, 2), (67, 1, 14392, 1, 1, 4),
    (5, 1, 3707, 207, 9, 4), (97, 1, 11557, 2, 2, 4), (10, 1, 427, 736, 32, 4), (5, 1, 846, 704, 32, 4), (112, 1, 1653, 20, 1, 4), (2, 1, 2104, 720, 30, 4), (32, 56, 56, 256, 32, 2),
    (600, 1, 1, 8191, 1, 4), (600, 1, 1, 8191, 1, 2), (600, 1, 1, 8184, 8, 4), (600, 1, 1, 8184, 8, 2), (600, 1, 1, 8188, 1, 4), (3, 5, 5, 8190, 2, 4), (40, 1, 30, 4100, 5, 2),
    (1, 1, 4200, 8192, 8192, 2), (600, 2, 1, 64, 8, 4), (600, 2, 1, 64, 8, 2), (600, 1, 3, 150, 10, 2), (5, 6, 7, 1024, 64, 2),
]


def test_the_cases_take_every_way_backward():
    loop, sweeps, both = 0, 0, 0
    for *shape, size in BACKWARD:
        held, V = _backward_path(shape, F32 if size == 4 else BF16)
        if not held:
            several, wide = shape[0] > norm_choice.chunks(shape, size)["images"], shape[3] // V > 512
            loop, sweeps, both = loop + several, sweeps + wide, both + (several and wide)
    assert loop >= 10 and sweeps >= 6 and both >= 5


def _backward_want(x, dy, stats, gamma, beta, res, act):
    """As in test_gpu_norm.py: the formulas in 64 bits with the statistics given, and bounds on what fp32 may do to them."""
    B, H, W, C = x.shape
    mean, rstd = (s.double() for s in stats)
    G = mean.shape[1]
    spread = lambda s: _spread(s, C)
    xhat, w = (x.double() - spread(mean)) * spread(rstd), gamma.double()
    pre = xhat * w + beta.double() + (0 if res is None else res.double())
    s = torch.sigmoid(pre)
    slope = {"none": torch.ones_like(pre), "relu": (pre > 0).double(), "silu": s * (1 + pre * (1 - s))}[act]
    d = dy.double() * slope
    per = lambda v: v.reshape(B, H * W, G, C // G).mean((1, 3))
    g = d * w
    m1, m2 = spread(per(g)), spread(per(g * xhat))
    dx = spread(rstd) * (g - m1 - xhat * m2)
    terms = (xhat * w).abs() + beta.double().abs() + (0 if res is None else res.double().abs())
    d_err = E * dy.double().abs() * (16 + (4 * terms + 8 * pre.abs() if act == "silu" else 0))
    g_err = d_err * w.abs() + 2 * E * g.abs()
    a1, a2 = spread(per(g.abs())), spread(per((g * xhat).abs()))
    e1, e2 = spread(per(g_err)) + 256 * E * a1, spread(per(g_err * xhat.abs())) + 260 * E * a2
    dx_err = spread(rstd) * (g_err + e1 + xhat.abs() * e2 + 8 * E * (g.abs() + m1.abs() + (xhat * m2).abs()))
    total = lambda v: v.sum((0, 1, 2))
    return pre, {"dx": (dx, dx_err), "dgamma": (total(d * xhat), total(d_err * xhat.abs()) + 260 * E * total((d * xhat).abs())),
                 "dbeta": (total(d), total(d_err) + 256 * E * total(d.abs())), "dresidual": (d, d_err)}


@pytest.mark.parametrize("case,dtype", _typed(BACKWARD))
def test_backward(case, dtype):
    shape = case[:5]
    B, H, W, C, G = shape
    act = ("silu", "none", "relu")[(B + C + H) % 3]
    print("[case] norm backward", shape, dtype, act, _backward_path(shape, dtype), flush=True)
    x, gamma, beta, res, g = _inputs(B, H, W, C, dtype, residual=(W + G) % 2 == 1, seed=6)
    dy = torch.randn((B, H, W, C), generator=g).to(dtype)
    x, gamma, beta, res, dy = x.cuda(), gamma.cuda(), beta.cuda(), None if res is None else res.cuda(), dy.cuda()
    _, _, mean, rstd = R.group_norm(x, G, EPS, gamma, beta, res)
    stats = (mean.float(), rstd.float())
    if act == "relu":      # next to the border of a ReLU its slope may be either: no gradient comes from there
        pre, _ = _backward_want(x, dy, stats, gamma, beta, res, act)
        dy = torch.where(pre.abs() < 1e-4 * (1 + x.double().abs().max() * rstd.max()), torch.zeros_like(dy), dy)
    gn = _layer(B, H, W, C, G, act, dtype)
    got = gn.backward(x, dy, stats, gamma, beta, residual=res)
    _, want = _backward_want(x, dy, stats, gamma, beta, res, act)
    for t, (name, (v, err)) in zip(got, want.items()):
        if name == "dresidual" and res is None:
            assert t is None
            continue
        R.assert_within(t, v.cpu(), err.cpu(), F32 if name in ("dgamma", "dbeta") else dtype, name)
    again = gn.backward(x, dy, stats, gamma, beta, residual=res)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


def test_slices_that_a_launch_has_no_threads_for():
    """65535 images of one pixel, 8144 = 16 * 509 channels in 509 groups in fp32: slices of 16 channels would need 2^33 threads, so
    that images go over chunks, several sweeps of a workgroup to a pixel."""
    B, C, G = 65535, 8144, 509
    gn = _layer(B, 1, 1, C, G, "relu")
    assert gn.kernel_count() == 2 and norm_choice.slices((B, 1, 1, C, G), 4, 4)["held"] == 0
    x = torch.empty((B, 1, 1, C), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(6))
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    y = gn(x, gamma, beta)
    some = torch.tensor([0, 1, 255, 30000, B - 2, B - 1], device="cuda")
    want, _, _, bound = _forward_want(x[some], G, "relu", gamma, beta, None)
    R.assert_within(y[some], want.cpu(), bound.cpu(), F32, "y")
