"""Microscaled 4-bit floating point for callers that hold torch tensors (``include/tdc_mx4.h``): quantisation, products, and
1x1 convolutions with weights in 4 bits.

A quantised tensor is a pair (codes, scales): of a tensor [...][C], codes are uint8 [...][16 * ceil(C/32)] (two values to a
byte) and scales uint8 [...][ceil(C/32)], one power of two to a block of 32.  Marshalling only; the arithmetic is in libtdc.so.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from ._tensors import act_code, dtype_code, expect, on_stream, pixel_pitch, sizes, stream_handle, torch_stream
from .layer import _order_after


def _call(fn, device, stream, *args, name):
    """A call without a plan runs on the current device: make it the tensors'."""
    import torch
    if torch.cuda.current_device() == device.index:
        rc = fn(stream_handle(stream, device), *args)
    else:
        with torch.cuda.device(device):
            rc = fn(stream_handle(stream, device), *args)
    if rc:
        raise B.TdcError(rc, name)


def _row_pitch(x):
    """x [..., C] as rows of C values at an even distance: that distance."""
    if x.is_contiguous():
        return x.shape[-1]
    if x.dim() > 1 and x.stride(-1) == 1 or x.shape[-1] == 1:
        pitch, span = None, 0
        for size, stride in reversed(list(zip(x.shape[:-1], x.stride()[:-1]))):
            if size == 1:
                continue
            if pitch is None:
                pitch, span = stride, stride * size
            elif stride != span:
                pitch = -1
                break
            else:
                span = stride * size
        if pitch is None:
            return x.shape[-1]
        if pitch >= x.shape[-1]:
            return pitch
    raise ValueError("x must have its last dimension's values next to each other and its rows evenly spaced, not strides %s" % (tuple(x.stride()),))


def _rows(shape) -> int:
    n = 1
    for s in shape:
        n *= s
    return n


def quantize(x, stream=None):
    """(codes, scales) of x [..., C], float32, float16 or bfloat16."""
    import torch
    code = dtype_code(x.dtype)
    if not x.is_cuda or x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be a tensor on a GPU with a last dimension of at least one value")
    C, lead, device = x.shape[-1], x.shape[:-1], x.device
    nb, pitch = -(-C // 32), _row_pitch(x)
    with on_stream(stream, device, (x,)):
        codes = torch.empty(lead + (nb * 16,), device=device, dtype=torch.uint8)
        scales = torch.empty(lead + (nb,), device=device, dtype=torch.uint8)
    _call(B.load().tdc_mx4_quantize, device, stream, x.data_ptr(), code, x.numel() // C, C, pitch, codes.data_ptr(), scales.data_ptr(), name="tdc_mx4_quantize")
    return codes, scales


def _pair(codes, scales, C, name):
    """Checks a quantised tensor of rows of C values; returns its leading dimensions."""
    import torch
    nb, lead = -(-C // 32), codes.shape[:-1]
    if not codes.is_cuda:
        raise ValueError("%s must be on a GPU" % name)
    expect(codes, name + " codes", lead + (nb * 16,), torch.uint8, codes.device)
    expect(scales, name + " scales", lead + (nb,), torch.uint8, codes.device)
    return lead


def dequantize(codes, scales, C: int, dtype=None, stream=None):
    """The values [..., C] that (codes, scales) stand for, rounded to ``dtype`` (default float32)."""
    import torch
    if C < 1:
        raise ValueError("C must be at least 1")
    dtype = dtype or torch.float32
    lead, code, device = _pair(codes, scales, C, "x"), dtype_code(dtype), codes.device
    with on_stream(stream, device, (codes, scales)):
        y = torch.empty(lead + (C,), device=device, dtype=dtype)
    _call(B.load().tdc_mx4_dequantize, device, stream, codes.data_ptr(), scales.data_ptr(), _rows(lead), C, y.data_ptr(), code, 0, name="tdc_mx4_dequantize")
    return y


def matmul(a, b, K: int, bias=None, residual=None, act: str = "none", dtype=None, y=None, stream=None):
    """y[..., N] = act(a b^T + bias + residual) for a = (codes, scales) of [..., K] and b of [N, K]; y in ``dtype`` (default float32)."""
    import torch
    if K < 1:
        raise ValueError("K must be at least 1")
    dtype = dtype or torch.float32
    code, lead, b_lead, dev = dtype_code(dtype), _pair(*a, K, "a"), _pair(*b, K, "b"), a[0].device
    if len(b_lead) != 1 or b[0].device != dev:
        raise ValueError("b must hold rows [N][K] on a's device")
    N, M = b_lead[0], _rows(lead)
    if max(M, N, K) >> 31:
        sizes(M=M, N=N, K=K)
    bias_p = None if bias is None else expect(bias, "bias", (N,), torch.float32, dev).data_ptr()
    res_p = None if residual is None else expect(residual, "residual", lead + (N,), dtype, dev).data_ptr()
    epi = B.tdc_mx4_epilogue(bias_p, res_p, act_code(act))
    with on_stream(stream, dev, tuple(a) + tuple(b) + (bias, residual, y)):
        y = torch.empty(lead + (N,), device=dev, dtype=dtype) if y is None else expect(y, "y", lead + (N,), dtype, dev)
    _call(B.load().tdc_mx4_matmul, dev, stream, a[0].data_ptr(), a[1].data_ptr(), b[0].data_ptr(), b[1].data_ptr(), M, N, K, y.data_ptr(), code, ctypes.byref(epi),
          name="tdc_mx4_matmul")
    return y


class MX4Conv2d:
    """A 1x1 convolution (any stride, no padding) on channels-last tensors with weights in 4 bits, bound to a device plan.

    Called with x [batch][H][W][C] in ``dtype``, which it quantises along C itself, or with a quantised pair of one row per input
    pixel (GroupNorm.quantized, quantize).  y [batch][Ho][Wo][N] in ``dtype``."""

    def __init__(self, layer, dtype=None, device: int = 0, x_pitch: int = 0):
        """``layer`` has fields batch, C, N, H, W, K, stride, pad (e.g. workloads.Layer) with K = 1 and pad = 0.
        ``x_pitch``: elements from one input pixel to the next (default C), for an x that is a slice of wider pixels."""
        import torch
        self.plan = None
        if layer.K != 1 or layer.pad != 0:
            raise ValueError("a 4-bit convolution is 1x1 without padding")
        sizes(**{k: getattr(layer, k) for k in ("batch", "H", "W", "C", "N", "stride")})
        self.layer, self.dtype = layer, dtype or torch.float32
        self.dev = torch.device("cuda", device)
        self.x_pitch = x_pitch or layer.C
        self._pack_event = None
        self.plan = B.tdc_mx4_plan_create(B.tdc_mx4_shape(layer.batch, layer.H, layer.W, layer.C, layer.N, layer.stride, dtype_code(self.dtype), self.x_pitch), device)
        self._in, self._out = (layer.batch, layer.H, layer.W, layer.C), (layer.batch, (layer.H - 1) // layer.stride + 1, (layer.W - 1) // layer.stride + 1, layer.N)

    def out_shape(self):
        return self._out

    def kernel_count(self) -> int:
        return B.tdc_mx4_plan_kernel_count(self.plan)

    def pack(self, W, stream=None) -> None:
        """Quantise W [C][N][1][1] (or [C][N]), float32, into the plan, once.  W is not needed afterwards.

        Runs on ``stream`` (default: the current stream); a later call on another stream is made to wait for it."""
        import torch
        L = self.layer
        if tuple(W.shape) not in ((L.C, L.N, 1, 1), (L.C, L.N)):
            raise ValueError("W must be [%d][%d][1][1], not %s" % (L.C, L.N, tuple(W.shape)))
        expect(W, "W", W.shape, torch.float32, self.dev)
        with on_stream(stream, self.dev, (W,)):
            B.tdc_mx4_plan_pack(self.plan, W, stream_handle(stream, self.dev))
        ts = torch_stream(stream, self.dev)
        self._pack_event = ts.record_event()
        self._ordered = {ts.cuda_stream}

    def _arguments(self, x, y, bias, residual, act):
        import torch
        L = self.layer
        shape, out = self._in, self._out
        if isinstance(x, (tuple, list)):
            if _rows(_pair(*x, L.C, "x")) != L.batch * L.H * L.W or x[0].device != self.dev:
                raise ValueError("x must hold one row of %d values for each of %d pixels on %s" % (L.C, L.batch * L.H * L.W, self.dev))
            fn, ins = B.load().tdc_conv_mx4_quantized, (x[0].data_ptr(), x[1].data_ptr())
        else:
            pitch = pixel_pitch(x, "x", shape, self.dtype, self.dev)
            if pitch != self.x_pitch and L.batch * L.H * L.W > 1:
                raise ValueError("the layer was made for pixels %d elements apart, not %d" % (self.x_pitch, pitch))
            fn, ins = B.load().tdc_conv_mx4, (x.data_ptr(),)
        bias_p = None if bias is None else expect(bias, "bias", (L.N,), torch.float32, self.dev).data_ptr()
        res_p = None if residual is None else expect(residual, "residual", out, self.dtype, self.dev).data_ptr()
        code = act_code(act)
        epi = ctypes.byref(B.tdc_mx4_epilogue(bias_p, res_p, code)) if bias_p or res_p or code else None
        return fn, ins + (expect(y, "y", out, self.dtype, self.dev).data_ptr(), epi)

    def __call__(self, x, y=None, bias=None, residual=None, act: str = "none", stream=None):
        """y = act(conv(x) + bias[n] + residual)."""
        import torch
        if self._pack_event is not None:
            _order_after(self, torch_stream(stream, self.dev))
        if stream is not None:
            with on_stream(stream, self.dev, (tuple(x) if isinstance(x, (tuple, list)) else (x,)) + (bias, residual, y)):
                y = torch.empty(self._out, device=self.dev, dtype=self.dtype) if y is None else y
        elif y is None:
            y = torch.empty(self._out, device=self.dev, dtype=self.dtype)
        fn, args = self._arguments(x, y, bias, residual, act)
        rc = fn(self.plan, stream_handle(stream, self.dev), *args)
        if rc:
            raise B.TdcError(rc, "tdc_conv_mx4")
        return y

    def bind(self, x, y, bias=None, residual=None, act: str = "none", stream=None):
        """A zero-argument launcher with the arguments marshalled once.  The tensors and the stream must outlive it."""
        import torch
        if self._pack_event is not None:
            _order_after(self, torch_stream(stream, self.dev))
        fn, args = self._arguments(x, y, bias, residual, act)
        handle = ctypes.c_void_p(stream_handle(stream, self.dev))
        args = tuple(ctypes.c_void_p(a) if isinstance(a, int) else a for a in args)

        def launch():
            rc = fn(self.plan, handle, *args)          # keeps the layer, and refuses once it is closed
            if rc:
                raise B.TdcError(rc, "tdc_conv_mx4")

        return launch

    def close(self) -> None:
        if self.plan is not None:
            B.tdc_mx4_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
