"""Group norm at the ends of what it takes: the largest images, values that are no numbers, launches that differ from call to call.

Tolerances as in test_gpu_norm.py: E = 2^-24 to a rounding, counted below where a thread merges or adds up more than there."""
import pytest
import torch

import mx4_reference as R
import norm_choice
from test_gpu_norm import _inputs, _layer

pytestmark = pytest.mark.gpu
E = R.E24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _over(got, want, bound, dtype):
    """How far |got - want| passes the bound and half a step of dtype, on the GPU; both [n]."""
    return float(((got.double() - want).abs() - bound - (want.abs() + bound) * R.HALF[dtype]).max())


def test_an_image_next_to_2_31_pixels():
    """46340 x 46341 pixels, whose number added to a chunk's passes 2^31.  A thread has 4096 of them.  Forward it merges them by
    fours: 1024 roundings of the mean, and ten of differences that count less and less (the sum of 1/n, 8): 1200 E of the largest
    value with the levels behind.  Backward it adds them up one after another: 4096 additions, and under 200 behind those."""
    H, W = 46340, 46341
    c = norm_choice.chunks((1, H, W, 1, 1), 2)
    assert c["chunks"] == 1024 and norm_choice.slices((1, H, W, 1, 1), 2, 1)["held"] == 0
    g = torch.Generator(device="cuda").manual_seed(8)
    x, dy = (torch.empty((1, H, W, 1), device="cuda", dtype=BF16).normal_(generator=g) for _ in range(2))
    gamma, beta = torch.tensor([1.25], device="cuda"), torch.tensor([-0.5], device="cuda")
    gn = _layer(1, H, W, 1, 1, "none", BF16)
    stats = gn.new_stats()
    y = gn(x, gamma, beta, stats=stats)
    dx, dgamma, dbeta, _ = gn.backward(x, dy, stats, gamma, beta)
    pieces = lambda *ts: zip(*(t.reshape(-1).split(1 << 25) for t in ts))
    n, top = H * W, float(x.abs().max())
    mean = sum(float(a.double().sum()) for a, in pieces(x)) / n
    var = sum(float((a.double() - mean).square().sum()) for a, in pieces(x)) / n
    rstd = (var + 1e-5) ** -0.5
    assert abs(float(stats[0]) - mean) <= 1200 * E * top and abs(float(stats[1]) - rstd) <= 1200 * E * rstd
    w, b = float(gamma), float(beta)
    for a, got in pieces(x, y):
        xhat = (a.double() - mean) * rstd
        assert _over(got, xhat * w + b, E * (1200 * (xhat.abs() + top * rstd) * w + 48 * abs(b)), BF16) <= 0
    mean, rstd = float(stats[0]), float(stats[1])
    s1 = s2 = a1 = a2 = 0.0
    for a, d in pieces(x, dy):
        d, t = d.double(), (a.double() - mean) * rstd * d.double()
        s1, s2, a1, a2 = s1 + float(d.sum()), s2 + float(t.sum()), a1 + float(d.abs().sum()), a2 + float(t.abs().sum())
    assert abs(float(dbeta) - s1) <= 4300 * E * a1 and abs(float(dgamma) - s2) <= 4300 * E * a2
    for a, d, got in pieces(x, dy, dx):
        xhat = (a.double() - mean) * rstd
        want = rstd * w * (d.double() - s1 / n - xhat * s2 / n)
        bound = rstd * w * E * (4310 * (a1 + xhat.abs() * a2) / n + 16 * (d.double().abs() + xhat.abs()))
        assert _over(got, want, bound, BF16) <= 0


# one workgroup holds the image or a slice of it; an image in chunks
@pytest.mark.parametrize("shape", [(2, 8, 8, 32, 4), (2, 150, 201, 16, 4)], ids=["resident", "chunks"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_relu_chooses_gradients(shape, dtype):
    """An infinite dy behind a closed ReLU is as good as 0 there; a NaN before a ReLU reaches the gradients that its value enters,
    and no others."""
    B, H, W, C, G = shape
    assert (norm_choice.slices(shape, 4 if dtype is F32 else 2, 4, backward=True)["held"] > 0) == (H == 8)
    x, gamma, beta, res, g = _inputs(B, H, W, C, dtype, residual=False, seed=3)
    res = torch.randn((B, H, W, C), generator=g).to(dtype)
    dy = torch.randn((B, H, W, C), generator=g).to(dtype)
    res[1, 5, 3, 9] = -100                                    # closed
    res[0, 2, 2, 6] = 100                                     # open
    gn = _layer(B, H, W, C, G, "relu", dtype)
    stats = gn.new_stats()
    args = (x.cuda(), gamma.cuda(), beta.cuda())
    grads = lambda dy, res: [t.cpu() for t in gn.backward(args[0], dy.cuda(), stats, *args[1:], residual=res.cuda())]
    gn(*args, residual=res.cuda(), stats=stats)
    dy[1, 5, 3, 9] = 0
    want = grads(dy, res)
    assert all(bool(torch.isfinite(t).all()) for t in want) and float(want[3][1, 5, 3, 9]) == 0
    for bad in (float("inf"), -float("inf"), float("nan")):
        dy[1, 5, 3, 9] = bad
        assert all(torch.equal(a, b) for a, b in zip(grads(dy, res), want))
    dy[1, 5, 3, 9] = 0
    for where in ((1, 5, 3, 9), (0, 2, 2, 6)):
        holed = res.clone()
        holed[where] = float("nan")
        b, c = where[0], where[3]
        group = slice(c // (C // G) * (C // G), (c // (C // G) + 1) * (C // G))
        y = gn(*args, residual=holed.cuda()).cpu()
        assert bool(torch.isnan(y[where])) and int(torch.isnan(y).sum()) == 1
        dx, dgamma, dbeta, dres = grads(dy, holed)
        for got, good, at, count in ((dx, want[0], (b, slice(None), slice(None), group), H * W * C // G), (dgamma, want[1], c, 1), (dbeta, want[2], c, 1),
                                     (dres, want[3], where, 1)):
            nan = torch.isnan(got)
            assert bool(nan[at].all()) and int(nan.sum()) == count
            assert torch.equal(got[~nan], good[~nan])


@pytest.mark.parametrize("shape", [(2, 3, 3, 8191, 1), (2, 1, 1, 8190, 2), (1, 1, 4200, 8192, 8192)], ids=lambda s: "x".join(map(str, s)))
def test_launches_with_64_kib_of_lds_as_a_streams_first(shape):
    """The widest pixels in chunks, whose kernels take up to 68 KiB of LDS, captured before any such call ran."""
    B, H, W, C, G = shape
    assert norm_choice.slices(shape, 2, 1 if C % 2 else 2 if C % 4 else 4, backward=True)["held"] == 0
    xs = [torch.empty((B, H, W, C), device="cuda", dtype=BF16).normal_(generator=torch.Generator(device="cuda").manual_seed(s)) for s in (1, 2)]
    dy, gamma, beta = xs[1] * 0.5, torch.full((C,), 1.5, device="cuda"), torch.full((C,), 0.25, device="cuda")
    gn = _layer(B, H, W, C, G, "silu", BF16)
    stats, static = gn.new_stats(), torch.zeros_like(xs[0])

    def both(x):
        return (gn(x, gamma, beta, stats=stats),) + gn.quantized(x, gamma, beta) + gn.backward(x, dy, stats, gamma, beta)[:3]

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(static)
    for i in (0, 1, 0):
        static.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, both(xs[i]))), i
        torch.cuda.synchronize()


# resident; chunks; chunks of pixels with more pieces than threads, several images to a workgroup
GRADS = [(2, 8, 8, 32, 4), (2, 90, 110, 40, 5), (530, 1, 1, 8184, 8)]


@pytest.mark.parametrize("extra,offset", [(0, 0), (8, 8), (16, 4), (3, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", GRADS, ids=lambda s: "x".join(map(str, s)))
def test_gradients_into_slices_and_only_those_wanted(shape, dtype, extra, offset):
    """tdc_group_norm_backward with dx and dresidual in wider pixels, whose rest stays as it was, and without gradients that are not
    wanted: one statistic of the forward pass, dgamma or dbeta or neither, no dresidual, dresidual without a residual."""
    from paper_2211_03715_amd import binding as B
    from test_gpu_norm_paths import _backward_want
    n, H, W, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(C)
    randn = lambda *s: torch.randn(s, device="cuda", generator=g)
    x, dy, res = (randn(n, H, W, C).to(dtype) for _ in range(3))
    gamma, beta = 1 + 0.2 * randn(C), 0.2 * randn(C)
    gn = _layer(n, H, W, C, G, "silu", dtype)
    mean, rstd = gn.new_stats()
    alone = gn.new_stats()
    y = gn(x, gamma, beta, residual=res, stats=(mean, rstd))
    for kw in (dict(mean=alone[0]), dict(rstd=alone[1])):
        B.tdc_group_norm(gn.plan, x, gamma, beta, torch.empty_like(y), B.make_norm_args(residual=res, **kw))
    assert torch.equal(alone[0], mean) and torch.equal(alone[1], rstd)
    pitch = C + extra + offset
    cut = lambda t: t[..., offset:offset + C]

    def backward(dgamma=True, dbeta=True, dresidual=True, residual=True):
        wide = [torch.full((n, H, W, pitch), 7.0, device="cuda", dtype=dtype) for _ in range(2)]
        sums = [torch.full((C,), float("nan"), device="cuda") for _ in range(2)]
        B.tdc_group_norm_backward(gn.plan, x, dy, mean, rstd, gamma, beta, cut(wide[0]), sums[0] if dgamma else None, sums[1] if dbeta else None,
                                  B.make_norm_grad_args(residual=res if residual else None, dresidual=cut(wide[1]) if dresidual else None, dx_pitch=pitch, dresidual_pitch=pitch))
        for t in wide:
            assert bool((t[..., :offset] == 7).all()) and bool((t[..., offset + C:] == 7).all())
        return [cut(wide[0])] + sums + [cut(wide[1])]

    for residual in (True, False):
        full = backward(residual=residual)
        _, want = _backward_want(x, dy, (mean, rstd), gamma, beta, res if residual else None, "silu")
        for t, (name, (v, err)) in zip(full, want.items()):
            R.assert_within(t, v.cpu(), err.cpu(), F32 if name in ("dgamma", "dbeta") else dtype, name)
        for kw in (dict(dgamma=False), dict(dbeta=False), dict(dgamma=False, dbeta=False), dict(dresidual=False)):
            got = backward(residual=residual, **kw)
            for t, whole, name in zip(got, full, ("dx", "dgamma", "dbeta", "dresidual")):
                if kw.get(name, True):
                    # without dresidual pieces may be wider, and sums in another order
                    v, err = want[name]
                    R.assert_within(t, v.cpu(), err.cpu(), F32 if name in ("dgamma", "dbeta") else dtype, name)
                    assert "dresidual" in kw or torch.equal(t, whole), (kw, name)
                else:
                    assert bool((t == 7).all()) if name == "dresidual" else bool(torch.isnan(t).all())
