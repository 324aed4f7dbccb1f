"""What the torch wrappers of ``rope`` and ``kv4`` share: C functions by signature, strides,
streams, devices."""
from __future__ import annotations

import contextlib
import ctypes

from . import MOA_OK, MoaAttnError, _DTYPE_CODES, _stream_handle, _torch, lib

i64, vp, f32, ci, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_int, ctypes.c_size_t
_Strides3 = ctypes.c_int64 * 3


def function(name, argtypes, restype=ci):
    """The library's function ``name``, looked up at its first call."""
    def call(*args):
        f = call.f
        if f is None:
            f = getattr(lib, name)
            f.argtypes, f.restype = argtypes, restype
            call.f = f
        return f(*args)
    call.f = None
    call.__name__ = call.__qualname__ = name
    return call


def array(values):
    """A host array of int64, or None."""
    if values is None:
        return None
    return (ctypes.c_int64 * len(values))(*[int(x) for x in values])


def strides(t):
    """(batch, head, row) strides of a [B, H, N, d] tensor, or None.  A dimension of size 1 has
    no stride to keep to: 0."""
    if t is None:
        return None
    s, n = t.stride(), t.shape
    return _Strides3(s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0)


def ptr(t):
    return None if t is None else t.data_ptr()


def check_rows(name, t, shape=None):
    """t is a [B, H, N, d] device tensor with contiguous heads."""
    if t.dim() != 4 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must be [B, H, N, d]" + ("" if shape is None else f" = {tuple(shape)}")
                         + f", got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.stride(3) != 1 and t.shape[3] > 1 and t.numel():
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    if t.dtype not in _DTYPE_CODES:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}; use torch.float32 or torch.bfloat16")


def check_list(name, t, shape, dtype, device):
    """t is a contiguous device tensor of this shape and type."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {tuple(shape)} tensor of {dtype} on {device}")


def same_device(*tensors):
    d = None
    for t in tensors:
        if t is not None:
            if d is None:
                d = t.device
            elif t.device != d:
                raise ValueError(f"tensors on {d} and on {t.device} in one call")
    return d


def on(device):
    """Makes ``device`` current for a call, where it is not already."""
    if device.index == _torch.cuda.current_device():
        return contextlib.nullcontext()
    return _torch.cuda.device(device)


def handle(stream, t):
    return _stream_handle(stream, t)


def done(status):
    if status != MOA_OK:
        raise MoaAttnError(status)
