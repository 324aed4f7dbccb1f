"""What the torch wrappers of ``rope`` and ``kv4`` share.

Calls of a few microseconds on the GPU wait for their host side, so a wrapper tests its arguments
with as few attribute reads as it can and goes through the functions here, which find out what is
wrong, only when a test fails.  A wrapper that is given a ``stream`` calls itself with that stream current:
what it allocates then belongs to the stream, and memory that it frees is not used again while the
stream still works on it.
"""
from __future__ import annotations

import ctypes
import struct

from . import MOA_OK, MoaAttnError, _DTYPE_CODES, _torch as torch, lib

i64, vp, f32, ci, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_int, ctypes.c_size_t


class Function:
    """The library's function ``name``, looked up at its first call."""

    def __init__(self, name, argtypes, restype=ci):
        self.name, self.argtypes, self.restype, self.f = name, argtypes, restype, None

    def bind(self):
        f = getattr(lib, self.name)
        f.argtypes, f.restype = self.argtypes, self.restype
        self.f = f
        return f

    def __call__(self, *args):
        return (self.f or self.bind())(*args)


class Packed(Function):
    """The library's function ``name`` of a record of ``words`` (a struct format)."""

    def __init__(self, name, words):
        super().__init__(name, [vp])
        self.pack = struct.Struct(words).pack


def run(function, device, *words):
    """Calls a Packed status function with ``device`` (an index) current; raises on a rejected call."""
    f, record = function.f or function.bind(), function.pack(*words)
    if device == torch._C._cuda_getDevice():
        status = f(record)
    else:
        with torch.cuda.device(device):
            status = f(record)
    if status != MOA_OK:
        raise MoaAttnError(status)


def on_stream(stream, t):
    """A context with the given stream, one of t's device, as the current one."""
    if stream.device != t.device:
        raise ValueError(f"a stream of {stream.device} for tensors on {t.device}")
    return torch.cuda.stream(stream)


def new_like(x):
    """A contiguous tensor like x (empty_like takes a third less time than new_empty)."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def is_list(t, shape, dtype, device):
    """Whether t is a contiguous tensor of this shape and type on that device (an index)."""
    return t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous()


def check_list(name, t, shape, dtype, device):
    if not is_list(t, shape, dtype, device):
        raise ValueError(f"{name} must be a contiguous {tuple(shape)} tensor of {dtype} on device {device}, got "
                         f"{tuple(t.shape)}, {t.dtype}, {t.device}")


def check_rows(name, t, shape=None, dtype=None, device=None):
    """t is a [B, H, N, d] device tensor with contiguous heads (of this shape, type and device)."""
    if t.dim() != 4 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be [B, H, N, d]" + ("" if shape is None else f" = {tuple(shape)}")
                         + f", got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.get_device() != device:
        raise ValueError(f"tensors on devices {device} and {t.get_device()} in one call")
    if t.stride(3) != 1 and t.shape[3] > 1 and t.numel():
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    if t.dtype not in _DTYPE_CODES:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}; use torch.float32 or torch.bfloat16")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be of {dtype}, got {t.dtype}")


def workspace(ws, device):
    """(address, bytes) of a workspace tensor or None."""
    if ws is None:
        return 0, 0
    if ws.get_device() != device or not ws.is_contiguous():
        raise ValueError(f"the workspace must be a contiguous tensor on device {device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()
