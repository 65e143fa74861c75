"""Activations held in 8 bits between forward and backward (include/checkpoint8.h): the C names, and pack, which makes a
Checkpoint8 of a tensor.  TriMul.backward and residual_backward take one in the place of z, and
normrotate.norm_rotate writes and reads them itself.  Streams and devices as in attention.py."""
import ctypes

import torch

from . import trimul as _t
from .trimul import DTYPE_CODE, TORCH_DTYPE, TRI_MUL_BF16, TRI_MUL_F32, _check, _i32, _i64, _ptr, _vp, on_stream

_DTYPES = {torch.float32: TRI_MUL_F32, torch.bfloat16: TRI_MUL_BF16}


class Checkpoint8View(ctypes.Structure):
    """checkpoint8_view_t."""
    _fields_ = [("rows", _i64), ("n", _i64), ("ld", _i64), ("dtype", _i32), ("group", _i32)]


# name -> (restype, argtypes); the same order and meaning as include/checkpoint8.h
SIGNATURES = {
    "checkpoint8_pack": (ctypes.c_int, [ctypes.POINTER(Checkpoint8View), _vp, _vp, _vp, _vp]),
    "checkpoint8_unpack": (ctypes.c_int, [ctypes.POINTER(Checkpoint8View), _vp, _vp, _vp, _vp]),
}

_lib = None


def lib():
    """libtrimul.so with this module's signatures set."""
    global _lib
    if _lib is None:
        L = _t.lib()
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def checkpoint8_pack(view, x, codes, powers, stream=None):
    _check(lib().checkpoint8_pack(view, _ptr(x), _ptr(codes), _ptr(powers), _t._stream(stream)))


def checkpoint8_unpack(view, codes, powers, out, stream=None):
    _check(lib().checkpoint8_unpack(view, _ptr(codes), _ptr(powers), _ptr(out), _t._stream(stream)))


def _rows(name, t):
    """(rows, n, elements from one row to the next) of a tensor whose rows, along its last axis, are contiguous and evenly
    spaced."""
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dim() == 0:
        raise ValueError(f"{name} must have an axis")
    n = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // n if n else 0), n, n
    if not t.numel():
        return 0, n, n
    if n > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must have unit stride along its last axis")
    rows, ld, step = 1, n, None
    for length, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if length == 1:
            continue
        if step is None:
            ld = stride
        elif stride != step:
            raise ValueError(f"the rows of {name} must be evenly spaced (strides {t.stride()}); pass a contiguous copy")
        rows, step = rows * length, stride * length
    return rows, n, ld


class Checkpoint8:
    """A tensor in 8 bits: `codes` [..., n] int8, `powers` [..., ceil(n / group)] uint8, both contiguous, and the type it
    came from."""
    __slots__ = ("codes", "powers", "group", "dtype")

    def __init__(self, codes, powers, group, dtype):
        if not 8 <= group <= 256 or group % 8 or dtype not in _DTYPES:
            raise ValueError(f"group must be a multiple of 8 up to 256 and dtype float32 or bfloat16, not {group} and {dtype}")
        shape = codes.shape[:-1] + (-(-codes.shape[-1] // group),)
        if codes.dtype != torch.int8 or powers.dtype != torch.uint8 or powers.shape != shape or powers.device != codes.device:
            raise ValueError(f"codes must be int8 and powers uint8 {list(shape)} on {codes.device}, not {codes.dtype} and {powers.dtype} {list(powers.shape)} on {powers.device}")
        if not codes.is_contiguous() or not powers.is_contiguous():
            raise ValueError("codes and powers must be contiguous")
        self.codes, self.powers, self.group, self.dtype = codes, powers, group, dtype

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def unpack(self, dtype=None, out=None, stream=None):
        """The values it stands for (exact in either type): of type `dtype` ("f32" or "bf16", default the original's), or
        into out, whose rows may be further apart than n."""
        dt = self.dtype if dtype is None else TORCH_DTYPE[DTYPE_CODE[dtype]]
        with on_stream(self.device, stream) as s:
            if out is None:
                out = torch.empty(self.shape, dtype=dt, device=self.device)
            elif out.shape != self.shape or out.device != self.device or (dtype is not None and out.dtype != dt):
                raise ValueError(f"out must be a {list(self.shape)} tensor on {self.device}" + (f" of {dt}" if dtype is not None else ""))
            rows, n, ld = _rows("out", out)
            checkpoint8_unpack(Checkpoint8View(rows, n, ld, _DTYPES[out.dtype], self.group), self.codes, self.powers, out, s)
        return out


def pack(x, group=32, stream=None):
    """x (float32 or bfloat16, contiguous along its last axis, its rows evenly spaced) as a Checkpoint8 with a power of two
    for each `group` values of a row (a multiple of 8 up to 256; a row's last group may be shorter)."""
    rows, n, ld = _rows("x", x)
    if group < 1:
        raise ValueError("group must be positive")
    with on_stream(x.device, stream) as s:
        codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        powers = torch.empty(tuple(x.shape[:-1]) + (-(-n // group),), dtype=torch.uint8, device=x.device)
        checkpoint8_pack(Checkpoint8View(rows, n, ld, _DTYPES[x.dtype], group), x, codes, powers, s)
    return Checkpoint8(codes, powers, group, x.dtype)
