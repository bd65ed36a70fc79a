"""Group norm with an activation on channels-last tensors, for callers that hold torch tensors (``include/tdc_norm.h``).

Marshalling only; the arithmetic is in libtdc.so.  A layer holds a plan with a workspace: its calls, and the replays of graphs
that captured them, must follow one another on one stream.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from ._tensors import act_code, dtype_code, expect, on_stream, pixel_pitch, sizes, stream_handle


def _float32():
    import torch
    return torch.float32


class GroupNorm:
    """y = act(group_norm(x) * gamma + beta + residual) on x [batch][H][W][C] with C/groups neighbouring channels to a group.

    x, residual and y are of ``dtype`` (float32, float16, bfloat16) and may be slices of the channels of wider pixels; gamma, beta
    and the statistics are float32.  ``act``: "none", "relu" or "silu".  As with the other layers no call enters torch's graph of
    gradients: a result does not require one, and backward() is called by the program."""

    def __init__(self, batch: int, H: int, W: int, C: int, groups: int, eps: float = 1e-5, act: str = "none", dtype=None, device: int = 0):
        import torch
        self.plan = None
        sizes(batch=batch, H=H, W=W, C=C, groups=groups)
        self.dtype = dtype or torch.float32
        self.shape = (batch, H, W, C)
        self._blocks = -(-C // 32)
        self.groups = groups
        self.act = act_code(act)
        self.dev = torch.device("cuda", device)
        self.plan = B.tdc_norm_plan_create(B.tdc_norm_shape(batch, H, W, C, groups, dtype_code(self.dtype), self.act, eps), device)

    def kernel_count(self, quantized: bool = False) -> int:
        """Launches of a call, or of one to quantized(), on aligned tensors without gaps."""
        return B.tdc_norm_plan_mx4_kernel_count(self.plan) if quantized else B.tdc_norm_plan_kernel_count(self.plan)

    def new_stats(self):
        """Tensors that a call fills with the mean and 1/standard deviation of every group, for backward()."""
        import torch
        return tuple(torch.empty((self.shape[0], self.groups), device=self.dev, dtype=torch.float32) for _ in range(2))

    def new_quantized(self):
        """(codes, scales) for quantized(): rows of C values in 4 bits, see mx4.py."""
        import torch
        return tuple(torch.empty(self.shape[:3] + (self._blocks * n,), device=self.dev, dtype=torch.uint8) for n in (16, 1))

    def _channel(self, t, name):
        return None if t is None else expect(t, name, self.shape[3:], _float32(), self.dev).data_ptr()

    def _pixels(self, t, name):
        return (None, 0) if t is None else (t.data_ptr(), pixel_pitch(t, name, self.shape, self.dtype, self.dev))

    def _stats(self, stats):
        if stats is None:
            return None, None
        mean, rstd = stats
        return tuple(expect(t, n, (self.shape[0], self.groups), _float32(), self.dev).data_ptr() for t, n in ((mean, "mean"), (rstd, "rstd")))

    def _forward(self, x, gamma, beta, residual, stats, y=None, quantized=None):
        """The foreign function of a forward call and its arguments behind the stream, and what they refer to."""
        import torch
        C = self.shape[3]
        xp, x_pitch = self._pixels(x, "x")
        rp, r_pitch = self._pixels(residual, "residual")
        mean, rstd = self._stats(stats)
        if quantized is None:
            yp, y_pitch = self._pixels(y, "y")
            fn, out = B.load().tdc_group_norm, (yp,)
        else:
            codes, scales = quantized
            y_pitch = C
            fn = B.load().tdc_group_norm_mx4
            out = (expect(codes, "codes", self.shape[:3] + (self._blocks * 16,), torch.uint8, self.dev).data_ptr(),
                   expect(scales, "scales", self.shape[:3] + (self._blocks,), torch.uint8, self.dev).data_ptr())
        args = None
        if rp or mean or x_pitch != C or y_pitch != C:
            args = ctypes.byref(B.tdc_norm_args(rp, mean, rstd, x_pitch, r_pitch, y_pitch))
        return fn, (xp, self._channel(gamma, "gamma"), self._channel(beta, "beta")) + out + (args,)

    def __call__(self, x, gamma=None, beta=None, residual=None, y=None, stats=None, stream=None):
        """Returns y (a new contiguous tensor unless given).  ``stats``: new_stats(), filled for backward()."""
        import torch
        if stream is not None:
            with on_stream(stream, self.dev, (x, gamma, beta, residual, y) + tuple(stats or ())):
                y = torch.empty(self.shape, device=self.dev, dtype=self.dtype) if y is None else y
        elif y is None:
            y = torch.empty(self.shape, device=self.dev, dtype=self.dtype)
        fn, args = self._forward(x, gamma, beta, residual, stats, y)
        rc = fn(self.plan, stream_handle(stream, self.dev), *args)
        if rc:
            raise B.TdcError(rc, "tdc_group_norm")
        return y

    def quantized(self, x, gamma=None, beta=None, residual=None, out=None, stats=None, stream=None):
        """The same values in 4 bits, (codes, scales), quantised from float32 before any rounding to dtype."""
        with on_stream(stream, self.dev, (x, gamma, beta, residual) + tuple(out or ()) + tuple(stats or ())):
            out = out or self.new_quantized()
            fn, args = self._forward(x, gamma, beta, residual, stats, quantized=out)
            rc = fn(self.plan, stream_handle(stream, self.dev), *args)
        if rc:
            raise B.TdcError(rc, "tdc_group_norm_mx4")
        return out

    def _bound(self, fn, args, stream, name):
        handle = ctypes.c_void_p(stream_handle(stream, self.dev))
        args = tuple(ctypes.c_void_p(a) if isinstance(a, int) else a for a in args)

        def launch():
            rc = fn(self.plan, handle, *args)          # keeps the layer, and refuses once it is closed
            if rc:
                raise B.TdcError(rc, name)

        return launch

    def bind(self, x, y, gamma=None, beta=None, residual=None, stats=None, stream=None):
        """A zero-argument launcher with the arguments marshalled once.  The tensors and the stream must outlive it."""
        return self._bound(*self._forward(x, gamma, beta, residual, stats, y), stream, "tdc_group_norm")

    def bind_quantized(self, x, out, gamma=None, beta=None, residual=None, stats=None, stream=None):
        return self._bound(*self._forward(x, gamma, beta, residual, stats, quantized=out), stream, "tdc_group_norm_mx4")

    def backward(self, x, dy, stats, gamma=None, beta=None, residual=None, stream=None):
        """(dx, dgamma, dbeta, dresidual) from the statistics that the forward call filled.  gamma, beta and residual are the
        forward call's; dresidual is None without a residual."""
        import torch
        C = self.shape[3]
        if stats is None:
            raise ValueError("stats must be what the forward call filled")
        mean, rstd = self._stats(stats)
        with on_stream(stream, self.dev, (x, dy, gamma, beta, residual) + tuple(stats)):
            dx = torch.empty(self.shape, device=self.dev, dtype=self.dtype)
            dgamma, dbeta = torch.empty((2, C), device=self.dev, dtype=torch.float32).unbind(0)
            dres = None if residual is None else torch.empty(self.shape, device=self.dev, dtype=self.dtype)
        xp, x_pitch = self._pixels(x, "x")
        dyp, dy_pitch = self._pixels(dy, "dy")
        rp, r_pitch = self._pixels(residual, "residual")
        args = None
        if rp or x_pitch != C or dy_pitch != C:
            args = ctypes.byref(B.tdc_norm_grad_args(rp, None if dres is None else dres.data_ptr(), x_pitch, r_pitch, dy_pitch, 0, 0))
        rc = B.load().tdc_group_norm_backward(self.plan, stream_handle(stream, self.dev), xp, dyp, mean, rstd, self._channel(gamma, "gamma"),
                                              self._channel(beta, "beta"), dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), args)
        if rc:
            raise B.TdcError(rc, "tdc_group_norm_backward")
        return dx, dgamma, dbeta, dres

    def close(self) -> None:
        if self.plan is not None:
            B.tdc_norm_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
