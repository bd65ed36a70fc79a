"""Bottleneck blocks with group norm and 4-bit 1x1 convolutions: every stage against its definition in 64 bits on what the stage
before it really stored, replays of a captured block and network against eager calls, and products captured by themselves."""
import numpy as np
import pytest
import torch

import mx4_reference as R
from parity_util import assert_parity
from test_gpu_mx4 import _product
from test_gpu_norm import _check_forward

pytestmark = pytest.mark.gpu
F32 = torch.float32


def _block(batch, C, M, H, W, R1, R2, stride, C_out):
    from paper_2211_03715_amd.bottleneck import TuckerNormBottleneck, make_norm_block_weights
    w = make_norm_block_weights(C, M, R1, R2, 11, C_out, projection=stride != 1 or C_out != C)
    return TuckerNormBottleneck(batch, C, M, H, W, R1, R2, w, stride=stride, C_out=C_out), w


def _conv1x1(got, pair, W, what):
    K, N = W.shape[:2]
    wv = R.values(*R.quantize(torch.from_numpy(W).reshape(K, N).t()), K)
    v, err = _product(R.values(*pair, K).reshape(-1, K), wv, None, None, "none", K)
    R.assert_within(got.reshape(-1, N), v, err, F32, what)


# batch, C, M, H, W, R1, R2, stride, C_out
BLOCKS = [(1, 64, 16, 14, 14, 8, 8, 1, 64), (2, 48, 24, 9, 11, 16, 20, 1, 48), (2, 64, 32, 13, 14, 8, 8, 2, 128), (1, 64, 64, 20, 20, 24, 24, 1, 256), (1, 256, 64, 56, 56, 16, 16, 1, 256)]


@pytest.mark.parametrize("shape", BLOCKS, ids=lambda s: "x".join(map(str, s)))
def test_every_stage_of_a_block(orc, shape):
    batch, C, M, H, W, R1, R2, stride, C_out = shape
    print("[case] norm block", shape, flush=True)
    blk, w = _block(*shape)
    x = torch.randn((batch, H, W, C), generator=torch.Generator().manual_seed(5))
    y = blk(x.cuda())
    torch.cuda.synchronize()
    cpu = lambda t: t.detach().cpu()
    t = lambda k: torch.from_numpy(w[k])
    t1, n1, t2, t3 = (cpu(v) for v in (blk.t1, blk.n1, blk.t2, blk.t3))
    _conv1x1(t1, R.quantize(x), w["W1"], "t1")
    _check_forward(n1, t1, blk.norm1.groups, "relu", F32, t("g1"), t("b1"), None, "n1")
    want, _ = orc.conv_factored(orc.Shape(**blk.l2.asdict()), np.ascontiguousarray(n1.numpy().transpose(0, 3, 1, 2)), w["U_in"], w["core"], w["U_out"])
    assert_parity(t2.numpy().transpose(0, 3, 1, 2), want, "t2 " + blk.describe())
    q2 = tuple(cpu(v) for v in blk.q2)
    normed = cpu(blk.norm2(blk.t2, blk.w["g2"], blk.w["b2"]))
    _check_forward(normed, t2, blk.norm2.groups, "relu", F32, t("g2"), t("b2"), None, "n2")
    assert all(torch.equal(a, b) for a, b in zip(q2, R.quantize(normed)))
    _conv1x1(t3, q2, w["W3"], "t3")
    shortcut = x
    if blk.projection:
        tp, shortcut = cpu(blk.tp), cpu(blk.s)
        _conv1x1(tp, tuple(v[:, ::stride, ::stride] for v in R.quantize(x)), w["Wp"], "tp")
        _check_forward(shortcut, tp, blk.normp.groups, "none", F32, t("gp"), t("bp"), None, "s")
    _check_forward(cpu(y), t3, blk.norm3.groups, "relu", F32, t("g3"), t("b3"), shortcut, "y")
    blk.close()


@pytest.mark.parametrize("shape", BLOCKS[1:3], ids=lambda s: "x".join(map(str, s)))
def test_a_captured_block(shape):
    blk, _ = _block(*shape)
    xs = [torch.randn((shape[0], shape[3], shape[4], shape[1]), generator=torch.Generator().manual_seed(s)).cuda() for s in range(3)]
    want = [blk(x).clone() for x in xs]
    static = torch.zeros_like(xs[0])
    graph = blk.capture(static)
    for i in (1, 0, 2, 1):
        static.copy_(xs[i])
        blk.y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(blk.y, want[i]), i
        assert torch.equal(blk(xs[(i + 1) % 3]), want[(i + 1) % 3])
        torch.cuda.synchronize()
    blk.close()


def test_a_network_of_such_blocks():
    """Block after block equals the same blocks called by hand, and so do replays of the whole."""
    from paper_2211_03715_amd import binding as B
    from paper_2211_03715_amd.bottleneck import TuckerResNetBody
    net = TuckerResNetBody(2, 17, 18, 32, blocks=(2, 1, 2, 1), layout=B.LAYOUT_NHWC, norm=True)
    assert net.kernels() >= 6 * 6 and len(net.describe().splitlines()) == 6
    xs = [torch.randn(net.in_shape, generator=torch.Generator().manual_seed(s)).cuda() for s in range(2)]
    want = []
    for x in xs:
        want.append(net(x).clone())
        h = x
        for blk in net.blocks:
            h = blk(h.clone())
        assert torch.equal(h, want[-1]) and bool(torch.isfinite(h).all()) and tuple(h.shape) == (2, 3, 3, 1024)
    static = torch.zeros_like(xs[0])
    graph = net.capture(static)
    for i in (1, 0, 1):
        static.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(net.y, want[i])
        assert torch.equal(net(xs[1 - i]), want[1 - i])
        torch.cuda.synchronize()
    net.close()


def test_blocks_with_channels_first_are_refused():
    from paper_2211_03715_amd import binding as B
    from paper_2211_03715_amd.bottleneck import TuckerNormBottleneck, make_norm_block_weights
    with pytest.raises(ValueError):
        TuckerNormBottleneck(1, 16, 8, 4, 4, 4, 4, make_norm_block_weights(16, 8, 4, 4, 0), layout=B.LAYOUT_NCHW)


@pytest.mark.parametrize("M,N,K", [(1, 300, 40000), (5, 64, 100), (200, 200, 256), (1500, 1300, 512), (2600, 3300, 128)])
def test_products_in_a_graph(M, N, K):
    """Quantisation, a product and dequantisation captured without a call of that size before them."""
    from paper_2211_03715_amd import mx4
    g = torch.Generator().manual_seed(M)
    b = mx4.quantize(torch.randn((N, K), generator=g).cuda())
    xs = [torch.randn((M, K), generator=g).half().cuda() for _ in range(2)]
    static = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = mx4.quantize(static)
        out = mx4.matmul(q, b, K, act="relu", dtype=torch.float16), mx4.dequantize(*q, K, dtype=torch.float16)
    for i in (0, 1, 0):
        static.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        p = mx4.quantize(xs[i])
        assert torch.equal(out[0], mx4.matmul(p, b, K, act="relu", dtype=torch.float16)) and torch.equal(out[1], mx4.dequantize(*p, K, dtype=torch.float16))


def _kernel_nodes(enqueue):
    """Kernels of a HIP graph that captures enqueue(): counted by the runtime."""
    import ctypes

    from paper_2211_03715_amd import binding as B
    lib = B.load()                                     # its dependencies' functions are found through it
    enqueue()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        enqueue()
    handle, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert lib.hipGraphGetNodes(handle, None, ctypes.byref(n)) == 0
    nodes, kinds = (ctypes.c_void_p * n.value)(), []
    assert lib.hipGraphGetNodes(handle, nodes, ctypes.byref(n)) == 0
    for node in nodes:
        kind = ctypes.c_int()
        assert lib.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        kinds.append(kind.value)
    return kinds.count(0)                              # hipGraphNodeTypeKernel


@pytest.mark.parametrize("shape", BLOCKS + [(32, 256, 64, 56, 56, 16, 16, 1, 256)], ids=lambda s: "x".join(map(str, s)))
def test_a_block_counts_its_launches(shape):
    """Against the kernels of its graph: at 56 x 56 the norm in 4 bits takes more launches than the same norm in fp32."""
    blk, _ = _block(*shape)
    x = torch.randn((shape[0], shape[3], shape[4], shape[1]), device="cuda")

    def run():
        blk.bind(x)
        blk()

    assert _kernel_nodes(run) == blk.kernels()
    blk.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 56, 56, 64, 32), (32, 56, 56, 64, 32), (2, 7, 7, 512, 32), (2, 9, 9, 40, 5), (1, 224, 224, 64, 32), (8, 28, 28, 128, 32)], ids=lambda s: "x".join(map(str, s)))
def test_a_norm_counts_its_launches(shape, dtype):
    from paper_2211_03715_amd.norm import GroupNorm
    gn = GroupNorm(*shape, dtype=dtype)
    x = torch.randn(shape[:4], device="cuda").to(dtype)
    y, q = torch.empty_like(x), gn.new_quantized()
    assert _kernel_nodes(lambda: gn(x, y=y)) == gn.kernel_count()
    assert _kernel_nodes(lambda: gn.quantized(x, out=q)) == gn.kernel_count(quantized=True)


def _stays(call, make):
    """What make() gives call() stays the call's until the stream it runs on is done, although the caller drops it at once."""
    side, busy = torch.cuda.Stream(), torch.empty(1 << 30, device="cuda")
    kept = make()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):                            # some 10 ms of work before the call's
            busy.fill_(1.0)
    call(kept, side)
    at = [t.data_ptr() for t in kept]
    sizes = [(t.shape, t.dtype) for t in kept]
    del kept
    new = [torch.empty(s, device="cuda", dtype=d) for s, d in sizes for _ in range(3)]
    assert not side.query(), "the stream was done too soon to tell"
    assert not set(at) & {t.data_ptr() for t in new}
    torch.cuda.synchronize()


def test_outputs_passed_in_are_kept_for_the_stream():
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.norm import GroupNorm
    from paper_2211_03715_amd.workloads import Layer
    x = torch.randn((2, 40, 40, 64), device="cuda")
    gn, conv = GroupNorm(2, 40, 40, 64, 8), mx4.MX4Conv2d(Layer(2, 64, 96, 40, 40, 1, 1, 1, 1, 0))
    conv.pack(torch.randn((64, 96), device="cuda"))
    a, b = mx4.quantize(x.reshape(-1, 64)), mx4.quantize(torch.randn((96, 64), device="cuda"))
    gn(x), gn.quantized(x), conv(x), mx4.matmul(a, b, 64)
    y, z = lambda: torch.empty_like(x), lambda: torch.empty(conv.out_shape(), device="cuda")
    _stays(lambda t, s: gn(x, y=t[0], stream=s), lambda: [y()])
    _stays(lambda t, s: gn(x, stats=tuple(t), stream=s), lambda: list(gn.new_stats()))
    _stays(lambda t, s: gn.quantized(x, out=tuple(t), stream=s), lambda: list(gn.new_quantized()))
    _stays(lambda t, s: gn.quantized(x, stats=tuple(t), stream=s), lambda: list(gn.new_stats()))
    _stays(lambda t, s: conv(x, t[0], stream=s), lambda: [z()])
    _stays(lambda t, s: conv(a, t[0], stream=s), lambda: [z()])
    _stays(lambda t, s: mx4.matmul(a, b, 64, y=t[0], stream=s), lambda: [z().reshape(-1, 96)])


def test_refusals_with_a_stream():
    """The same errors as without one."""
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.norm import GroupNorm
    from paper_2211_03715_amd.workloads import Layer
    side = torch.cuda.Stream()
    x, w = torch.zeros((2, 4, 4, 64), device="cuda"), torch.zeros(64, device="cuda")
    gn, conv = GroupNorm(2, 4, 4, 64, 8), mx4.MX4Conv2d(Layer(2, 64, 32, 4, 4, 1, 1, 1, 1, 0))
    conv.pack(torch.zeros((64, 32), device="cuda"))
    codes, scales = mx4.quantize(x.reshape(-1, 64))
    stats = gn.new_stats()
    for s in (None, side):
        for call in (lambda: gn(x.cpu(), stream=s), lambda: gn(x, w.cpu(), stream=s), lambda: gn(x, y=x.cpu(), stream=s), lambda: gn(x, stats=tuple(t.cpu() for t in stats), stream=s),
                     lambda: gn.quantized(x, out=(codes.cpu(), scales), stream=s), lambda: gn.backward(x, x.cpu(), stats, stream=s), lambda: gn.backward(x, x, None, stream=s),
                     lambda: mx4.dequantize(codes, scales.cpu(), 64, stream=s), lambda: mx4.matmul((codes, scales), (codes, scales.cpu()), 64, stream=s),
                     lambda: conv(x.cpu(), stream=s), lambda: conv(x, bias=torch.zeros(32), stream=s), lambda: conv(x, torch.zeros(conv.out_shape()), stream=s)):
            with pytest.raises(ValueError):
                call()
    torch.cuda.synchronize()
