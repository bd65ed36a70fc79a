"""Checks and marshalling of torch tensors for the layers of norm.py and mx4.py."""
from __future__ import annotations

from . import binding as B


_codes = {}


def dtype_code(dtype) -> int:
    if not _codes:
        import torch
        _codes.update({torch.float32: B.F32, torch.float16: B.F16, torch.bfloat16: B.BF16})
    code = _codes.get(dtype)
    if code is None:
        raise ValueError("dtype must be torch.float32, float16 or bfloat16, not %s" % (dtype,))
    return code


def act_code(act: str) -> int:
    if act not in B.ACTS:
        raise ValueError("act must be one of %s, not %r" % (sorted(B.ACTS), act))
    return B.ACTS[act]


def sizes(**named):
    """Sizes that go to the library in 32 bits, which would silently be cut to them."""
    for name, v in named.items():
        if not -2 ** 31 <= v < 2 ** 31:
            raise ValueError("%s must be below 2^31, not %d" % (name, v))


def _refuse(t, name, shape, dtype, device):
    raise ValueError("%s must be %s %s on %s, not %s %s on %s" % (name, tuple(shape), dtype, device, tuple(t.shape), t.dtype, t.device))


def expect(t, name: str, shape, dtype, device):
    """t is a contiguous tensor of that shape, dtype and device; returns it."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        _refuse(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def pixel_pitch(t, name: str, shape, dtype, device) -> int:
    """Elements from one pixel to the next of t [B][H][W][C], which may be a slice of the channels of wider pixels."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        _refuse(t, name, shape, dtype, device)
    if t.is_contiguous():
        return shape[-1]
    b, h, w, c = shape
    s = t.stride()
    pitch = s[2] if w > 1 else s[1] if h > 1 else s[0] if b > 1 else c
    if (c > 1 and s[3] != 1) or (h > 1 and s[1] != w * pitch) or (b > 1 and s[0] != h * w * pitch) or pitch < c:
        raise ValueError("%s must have its channels next to each other and its pixels evenly spaced, not strides %s" % (name, s))
    return pitch


def stream_handle(stream, device) -> int:
    """The raw handle of a stream; None is the current stream of the TENSORS' device, whichever device is current."""
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device.index)   # what current_stream(device).cuda_stream is, without the objects
    return stream if isinstance(stream, int) else stream.cuda_stream


def torch_stream(stream, device):
    """torch's stream object on `device` for None (its current stream), a raw handle (0: the default stream) or a torch stream."""
    import torch
    if stream is None:
        return torch.cuda.current_stream(device)
    if isinstance(stream, int):
        return torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    return stream


class on_stream:
    """New outputs are allocated, and what the caller passes is kept, for the stream that the call runs on:
    with on_stream(stream, device, tensors): ..."""

    def __init__(self, stream, device, tensors):
        self.context = None
        if stream is None:
            return
        import torch
        ts = torch_stream(stream, device)
        if ts.cuda_stream == torch.cuda.current_stream(device).cuda_stream:
            return
        if not torch.cuda.is_current_stream_capturing():
            for t in tensors:
                if t is not None and t.is_cuda:        # others are refused by the checks that follow
                    t.record_stream(ts)
        self.context = torch.cuda.stream(ts)

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()

    def __exit__(self, *exc):
        if self.context is not None:
            self.context.__exit__(*exc)
