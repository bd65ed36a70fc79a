"""Group norm and 4-bit products without a GPU: refusals come before any device call, struct layouts match the headers, and the
64-bit references agree with hand-worked values and with differences."""
import ctypes

import pytest
import torch

import mx4_reference as R
from paper_2211_03715_amd import binding as B

P = ctypes.c_void_p(4096)          # an address that is never read
ODD = ctypes.c_void_p(4097)


def test_struct_layouts():
    assert ctypes.sizeof(B.tdc_norm_shape) == 32 and ctypes.sizeof(B.tdc_norm_args) == 48 and ctypes.sizeof(B.tdc_norm_grad_args) == 56
    assert ctypes.sizeof(B.tdc_mx4_shape) == 40 and ctypes.sizeof(B.tdc_mx4_epilogue) == 24


def _norm(**kw):
    d = dict(batch=1, H=2, W=2, C=8, groups=2, dtype=0, act=0, eps=1e-5)
    d.update(kw)
    return B.tdc_norm_shape(*(d[k] for k in ("batch", "H", "W", "C", "groups", "dtype", "act", "eps")))


def test_norm_plans_are_refused():
    lib, plan = B.load(), ctypes.c_void_p()
    make = lambda **kw: lib.tdc_norm_plan_create(ctypes.byref(plan), ctypes.byref(_norm(**kw)), 0)
    assert lib.tdc_norm_plan_create(None, ctypes.byref(_norm()), 0) == B.TDC_ERR_NULL
    assert lib.tdc_norm_plan_create(ctypes.byref(plan), None, 0) == B.TDC_ERR_NULL
    for bad in (dict(batch=0), dict(H=0), dict(W=-1), dict(C=0), dict(groups=0), dict(groups=3), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert make(**bad) == B.TDC_ERR_BAD_SHAPE and not plan.value, bad
    for bad in (dict(dtype=3), dict(dtype=-1), dict(act=3), dict(batch=65536), dict(C=16384), dict(H=65536, W=65536)):
        assert make(**bad) == B.TDC_ERR_UNSUPPORTED and not plan.value, bad
    assert lib.tdc_norm_plan_destroy(None) == B.TDC_OK and lib.tdc_norm_plan_workspace_bytes(None) == 0 and lib.tdc_norm_plan_kernel_count(None) == 0
    assert lib.tdc_group_norm(None, None, P, None, None, P, None) == B.TDC_ERR_NULL
    assert lib.tdc_group_norm_mx4(None, None, P, None, None, P, P, None) == B.TDC_ERR_NULL
    assert lib.tdc_group_norm_backward(None, None, P, P, P, P, None, None, P, P, P, None) == B.TDC_ERR_NULL


def test_quantisation_is_refused():
    q, d = B.load().tdc_mx4_quantize, B.load().tdc_mx4_dequantize
    assert q(None, P, 0, 0, 8, 0, P, P) == B.TDC_OK and d(None, P, P, 0, 8, P, 0, 0) == B.TDC_OK        # no rows, nothing to do
    for call in (lambda p, t, r, c, s, k: q(None, p, t, r, c, s, k, P), lambda p, t, r, c, s, k: d(None, k, P, r, c, p, t, s)):
        assert call(None, 0, 1, 8, 0, P) == B.TDC_ERR_NULL and call(P, 0, 1, 8, 0, None) == B.TDC_ERR_NULL
        assert call(P, 0, -1, 8, 0, P) == B.TDC_ERR_BAD_SHAPE and call(P, 0, 1, 0, 0, P) == B.TDC_ERR_BAD_SHAPE and call(P, 0, 1, 8, 7, P) == B.TDC_ERR_BAD_SHAPE
        assert call(P, 3, 1, 8, 0, P) == B.TDC_ERR_UNSUPPORTED and call(P, 3, 0, 8, 0, P) == B.TDC_ERR_UNSUPPORTED
        assert call(ODD, 1, 1, 8, 0, P) == B.TDC_ERR_UNSUPPORTED and call(P, 0, 1, 8, 0, ctypes.c_void_p(4104)) == B.TDC_ERR_UNSUPPORTED
        assert call(P, 0, 1, 1 << 31, 0, P) == B.TDC_ERR_UNSUPPORTED and call(P, 0, 1 << 40, 8, 0, P) == B.TDC_ERR_UNSUPPORTED
        assert call(P, 0, 1 << 62, 1 << 30, 0, P) == B.TDC_ERR_UNSUPPORTED


def test_products_are_refused():
    fn = B.load().tdc_mx4_matmul
    call = lambda a=P, sa=P, b=P, sb=P, M=4, N=4, K=32, y=P, t=0, e=None: fn(None, a, sa, b, sb, M, N, K, y, t, ctypes.byref(e) if e is not None else None)
    assert call(M=0) == B.TDC_OK
    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(y=None)):
        assert call(**bad) == B.TDC_ERR_NULL, bad
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(K=-5)):
        assert call(**bad) == B.TDC_ERR_BAD_SHAPE, bad
    for bad in (dict(t=3), dict(a=ctypes.c_void_p(4104)), dict(b=ODD), dict(y=ODD), dict(M=1 << 30, N=1 << 20), dict(K=0x7fffffff),
                dict(e=B.make_mx4_epilogue(act=3)), dict(e=B.make_mx4_epilogue(bias=4098)), dict(e=B.make_mx4_epilogue(residual=4098))):
        assert call(**bad) == B.TDC_ERR_UNSUPPORTED, bad


def _mx4(**kw):
    d = dict(batch=1, H=2, W=2, C=8, N=4, stride=1, dtype=0, x_pitch=0)
    d.update(kw)
    return B.tdc_mx4_shape(*(d[k] for k in ("batch", "H", "W", "C", "N", "stride", "dtype", "x_pitch")))


def test_convolution_plans_are_refused():
    lib, plan = B.load(), ctypes.c_void_p()
    make = lambda **kw: lib.tdc_mx4_plan_create(ctypes.byref(plan), ctypes.byref(_mx4(**kw)), 0)
    assert lib.tdc_mx4_plan_create(None, ctypes.byref(_mx4()), 0) == B.TDC_ERR_NULL and lib.tdc_mx4_plan_create(ctypes.byref(plan), None, 0) == B.TDC_ERR_NULL
    for bad in (dict(batch=0), dict(H=0), dict(W=0), dict(C=0), dict(N=0), dict(stride=0), dict(x_pitch=7), dict(x_pitch=-8)):
        assert make(**bad) == B.TDC_ERR_BAD_SHAPE and not plan.value, bad
    for bad in (dict(dtype=3), dict(C=0x7fffffff), dict(batch=65536, H=256, W=256), dict(batch=1 << 20, H=32, W=32, N=1 << 20)):
        assert make(**bad) == B.TDC_ERR_UNSUPPORTED and not plan.value, bad
    assert lib.tdc_mx4_plan_destroy(None) == B.TDC_OK and lib.tdc_mx4_plan_workspace_bytes(None) == 0 and lib.tdc_mx4_plan_kernel_count(None) == 0
    assert lib.tdc_mx4_plan_pack(None, None, P) == B.TDC_ERR_NULL and lib.tdc_conv_mx4(None, None, P, P, None) == B.TDC_ERR_NULL
    assert lib.tdc_conv_mx4_quantized(None, None, P, P, P, None) == B.TDC_ERR_NULL


def test_python_layers_refuse_what_is_not_on_a_gpu():
    from paper_2211_03715_amd import mx4
    with pytest.raises(ValueError):
        mx4.quantize(torch.zeros(2, 32))
    with pytest.raises(ValueError):
        mx4.quantize(torch.zeros(2, 32, dtype=torch.float64))
    with pytest.raises(ValueError):
        mx4.dequantize(torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.uint8), 32)
    from paper_2211_03715_amd.workloads import Layer
    with pytest.raises(ValueError):
        mx4.MX4Conv2d(Layer(1, 8, 8, 4, 4, 1, 1))


def test_reference_quantisation_by_hand():
    x = torch.zeros(2, 34, dtype=torch.float64)
    # largest 6: scale 1.  Ties at 1/4, 3/4, 5/4, 7/4, 5/2, 7/2, 5 go to 0, 1, 1, 2, 2, 4, 4.
    x[0, :9] = torch.tensor([6, .25, .75, -1.25, 1.75, 2.5, 3.5, 5, -.2])
    x[0, 32:] = torch.tensor([7.9, 1.0])              # largest in [4, 8): scale 1, 7.9 becomes 6
    x[1, 0] = float("inf")
    x[1, 33] = 2.0 ** -149                            # 2^(-149-2) is below the least scale, 2^-127
    codes, scales = R.quantize(x)
    assert scales.tolist() == [[127, 127], [255, 0]]
    v = R.values(codes, scales, 34)
    assert v[0, :9].tolist() == [6, 0, 1, -1, 2, 2, 4, 4, -0.0] and v[0, 32:].tolist() == [6, 1]
    assert bool(torch.isnan(v[1, :32]).all()) and v[1, 32:].tolist() == [0, 0]
    assert codes[0, :2].tolist() == [7, 2 + 16 * (8 + 2)]


def test_reference_norm_by_hand():
    x = torch.tensor([1., 3, 10, 10, 5, 7, 10, 14]).reshape(1, 1, 2, 4)      # groups of two channels: {1, 3, 5, 7}, {10, 10, 10, 14}
    pre, xhat, mean, rstd = R.group_norm(x, 2, 0.0)
    assert mean.tolist() == [[4, 11]] and torch.allclose(rstd, torch.tensor([[5.0 ** -.5, 3.0 ** -.5]], dtype=torch.float64))
    assert torch.allclose(xhat[0, 0, 0], torch.tensor([-3, -1, 0, 0], dtype=torch.float64) * rstd[0].repeat_interleave(2) + torch.tensor([0, 0, -1, -1]) * rstd[0, 1])


def test_more_outputs_than_2_to_the_24_are_refused():
    lib, plan = B.load(), ctypes.c_void_p()
    assert lib.tdc_mx4_matmul(None, P, P, P, P, 1, (1 << 24) + 1, 32, P, 0, None) == B.TDC_ERR_UNSUPPORTED
    assert lib.tdc_mx4_plan_create(ctypes.byref(plan), ctypes.byref(_mx4(N=(1 << 24) + 1)), 0) == B.TDC_ERR_UNSUPPORTED and not plan.value


def test_the_limits_that_the_header_states():
    """Refused right above them; right below, what is refused is a device that is not there."""
    lib, plan = B.load(), ctypes.c_void_p()
    q, d = lib.tdc_mx4_quantize, lib.tdc_mx4_dequantize
    for rows, cols in ((2 ** 31 - 127, 1), (2 ** 31 - 127, 32), (2 ** 30 - 63, 33), (2 ** 6, 2 ** 30), (2 ** 62, 2 ** 30)):
        assert q(None, P, 2, rows, cols, 0, P, P) == B.TDC_ERR_UNSUPPORTED and d(None, P, P, rows, cols, P, 2, 0) == B.TDC_ERR_UNSUPPORTED, (rows, cols)
    for M, N in ((2 ** 31 - 255, 1), (2 ** 30, 257), (2 ** 22, 2 ** 17), (2 ** 23, 2 ** 16)):
        assert lib.tdc_mx4_matmul(None, P, P, P, P, M, N, 32, P, 0, None) == B.TDC_ERR_UNSUPPORTED, (M, N)
    make = lambda **kw: lib.tdc_mx4_plan_create(ctypes.byref(plan), ctypes.byref(_mx4(**kw)), 1 << 20)
    for above in (dict(H=2 ** 29 - 31, W=1), dict(H=2 ** 15, W=2 ** 16), dict(H=2 ** 12, W=2 ** 11, N=2 ** 16), dict(H=2 ** 14, W=2 ** 13, C=481)):
        assert make(**above) == B.TDC_ERR_UNSUPPORTED and not plan.value, above
    for below in (dict(H=2 ** 29 - 32, W=1), dict(H=2 ** 31 - 1, W=1, stride=5), dict(H=2 ** 12, W=2 ** 11, N=2 ** 16 - 256), dict(H=2 ** 14, W=2 ** 13, C=480),
                  dict(batch=64, H=224, W=224, C=64, N=4096, dtype=2)):
        assert make(**below) == B.TDC_ERR_HIP and not plan.value, below


def test_raw_streams_belong_to_the_layers_device(monkeypatch):
    """A handle means a stream of the layer's device, whichever is current: when weights are packed on it and when a call waits for that."""
    import contextlib

    from paper_2211_03715_amd import mx4
    there = torch.device("cuda", 1)
    made = []

    class Stream:
        def __init__(self, kind, handle, device):
            self.kind, self.cuda_stream, self.device, self.waited = kind, handle, device, False
            made.append(self)

        def record_event(self):
            return self                                # is its own event, never done

        def query(self):
            return False

        def wait_event(self, event):
            self.waited = True

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream("raw", handle, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream("default", 0, device))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("current", 77, device))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    conv = mx4.MX4Conv2d.__new__(mx4.MX4Conv2d)
    conv.plan, conv.dev, conv.dtype, conv._out = None, there, torch.float32, (1,)
    conv.layer = type("Layer", (), dict(C=8, N=4))
    conv._arguments = lambda *a: (lambda *b: B.TDC_OK, (None,))
    monkeypatch.setattr(mx4, "expect", lambda *a: None)
    monkeypatch.setattr(mx4, "on_stream", lambda *a: contextlib.nullcontext())
    monkeypatch.setattr(mx4.B, "tdc_mx4_plan_pack", lambda *a: None)
    y = torch.zeros(1)
    for packed_on, kind in ((12345, "raw"), (0, "default")):
        del made[:]
        conv.pack(torch.zeros(8, 4), stream=packed_on)
        conv(None, y=y, stream=54321)
        conv.bind(None, None, stream=65432)
        used = [s for s in made if s.kind != "current"]
        assert [s.kind for s in used] == [kind, "raw", "raw"] and all(s.device == there for s in used) and [s.waited for s in used] == [False, True, True]
    from paper_2211_03715_amd import _tensors
    own = Stream("own", 5, there)
    assert _tensors.torch_stream(own, there) is own and _tensors.torch_stream(None, there).device == there


def test_sizes_beyond_32_bits_are_refused(monkeypatch):
    """ctypes would hand the library their low 32 bits: a plan for 7 pixels where 2^32 + 7 were meant."""
    from types import SimpleNamespace

    from paper_2211_03715_amd import mx4, norm
    reached = []
    monkeypatch.setattr(B, "tdc_norm_plan_create", lambda *a: reached.append(a))
    monkeypatch.setattr(B, "tdc_mx4_plan_create", lambda *a: reached.append(a))
    for v in (2 ** 31, 2 ** 32 + 8):
        for i in range(5):
            args = [1, 8, 8, 8, 8]
            args[i] = v
            with pytest.raises(ValueError):
                norm.GroupNorm(*args)
        for name in ("batch", "H", "W", "C", "N", "stride"):
            layer = SimpleNamespace(**dict(dict(batch=1, H=8, W=8, C=8, N=8, stride=1, K=1, pad=0), **{name: v}))
            with pytest.raises(ValueError):
                mx4.MX4Conv2d(layer)
    # rows of a product: tensors that only say how large they are
    monkeypatch.setattr(mx4, "_pair", lambda codes, scales, K, name: codes.shape[:-1])
    large = SimpleNamespace(shape=(2 ** 16, 2 ** 16 + 1, 16), device="cuda:0")
    small = SimpleNamespace(shape=(4, 16), device="cuda:0")
    monkeypatch.setattr(mx4, "_call", lambda *a, **k: reached.append(a))
    for a, b, K in ((large, small, 32), (small, small, 2 ** 32 + 32)):
        with pytest.raises(ValueError):
            mx4.matmul((a, a), (b, b), K)
    assert not reached


def test_launchers_keep_their_layer_and_refuse_once_it_is_closed(monkeypatch):
    """A plan that went with its layer would be read after it was freed."""
    import gc

    from paper_2211_03715_amd import mx4, norm
    destroyed = []
    monkeypatch.setattr(B, "tdc_norm_plan_destroy", lambda plan: destroyed.append(plan.value))
    monkeypatch.setattr(B, "tdc_mx4_plan_destroy", lambda plan: destroyed.append(plan.value))
    monkeypatch.setattr(norm, "stream_handle", lambda *a: 0)
    monkeypatch.setattr(mx4, "stream_handle", lambda *a: 0)
    call = lambda plan, *a: B.TDC_ERR_NULL if plan is None else B.TDC_OK

    def made(cls, number):
        layer = cls.__new__(cls)
        layer.plan, layer.dev = ctypes.c_void_p(number), torch.device("cuda", 0)
        return layer

    def conv(number):
        layer = made(mx4.MX4Conv2d, number)
        layer._pack_event, layer._arguments = None, lambda *a: (call, (None,))
        return layer.bind(None, None), layer

    def gn(number):
        layer = made(norm.GroupNorm, number)
        layer._forward = lambda *a, **k: (call, (None,))
        return layer.bind(None, None), layer

    for make, number in ((conv, 1), (gn, 2)):
        launch = make(number)[0]
        gc.collect()
        assert number not in destroyed
        launch()
        launch, layer = make(10 + number)
        layer.close()
        assert destroyed[-1] == 10 + number
        with pytest.raises(B.TdcError):
            launch()


def test_a_stride_of_zero_is_the_plans_refusal():
    from paper_2211_03715_amd import mx4
    from paper_2211_03715_amd.workloads import Layer
    for stride in (0, -1):
        with pytest.raises(B.TdcError) as refused:
            mx4.MX4Conv2d(Layer(1, 8, 8, 4, 4, 1, 1, 1, stride, 0))
        assert refused.value.status == B.TDC_ERR_BAD_SHAPE
