"""Residual addition with dropout (include/pair_dropout.h): the C names, and dropout_add / dropout_backward, which
check their tensors and allocate outputs with torch.  The mask is a function of seed, offset and the element's place;
nothing of it is stored.  A captured call keeps its seed and offset: every replay drops the same elements.  Streams and
devices as in attention.py."""
import ctypes

import torch

from . import trimul as _t
from .trimul import DTYPE_CODE, TRI_MUL_BF16, TRI_MUL_F32, _check, _i32, _i64, _ptr, _vp, on_stream

PAIR_DROPOUT_EACH, PAIR_DROPOUT_ROWS, PAIR_DROPOUT_COLUMNS = 0, 1, 2
SHARE = {"none": PAIR_DROPOUT_EACH, "rows": PAIR_DROPOUT_ROWS, "columns": PAIR_DROPOUT_COLUMNS}
_DTYPES = {torch.float32: TRI_MUL_F32, torch.bfloat16: TRI_MUL_BF16}


class PairDropoutView(ctypes.Structure):
    """pair_dropout_view_t."""
    _fields_ = [("rows", _i64), ("cols", _i64), ("channels", _i64), ("row0", _i64), ("col0", _i64), ("n_cols", _i64),
                ("ld_x", _i64), ("ld_out", _i64), ("x_dtype", _i32), ("out_dtype", _i32), ("share", _i32),
                ("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


# name -> (restype, argtypes); the same order and meaning as include/pair_dropout.h
SIGNATURES = {
    "pair_dropout_add": (ctypes.c_int, [ctypes.POINTER(PairDropoutView), _vp, _vp, _vp, _vp]),
    "pair_dropout_backward": (ctypes.c_int, [ctypes.POINTER(PairDropoutView), _vp, _vp, _vp]),
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


def pair_dropout_add(view, x, res, out, stream=None):
    _check(lib().pair_dropout_add(view, _ptr(x), _ptr(res), _ptr(out), _t._stream(stream)))


def pair_dropout_backward(view, dout, dx, stream=None):
    _check(lib().pair_dropout_backward(view, _ptr(dout), _ptr(dx), _t._stream(stream)))


def _rows(name, t, shape=None, device=None):
    """Row stride of a [rows][cols][channels] tensor whose rows are contiguous."""
    n = t.shape
    if len(n) != 3 or (shape is not None and n != shape):
        raise ValueError(f"{name} must be [rows][cols][channels]" + (f" = {tuple(shape)}" if shape is not None else "") + f", not {list(n)}")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must live on {'the GPU' if device is None else device}")
    r, c, ch = n
    sr, sc, sch = t.stride()
    if ((ch > 1 and sch != 1) or (c > 1 and sc != ch)) and t.numel():
        raise ValueError(f"{name}'s columns and channels must be contiguous")
    return sr if r > 1 else c * ch


def _view(shape, ld_x, ld_out, x_dtype, out_dtype, p, seed, offset, share, row0, col0, n_cols):
    code = SHARE.get(share)
    if code is None:
        raise ValueError(f"share must be one of {sorted(SHARE)}, not {share!r}")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    rows, cols, channels = shape
    return PairDropoutView(rows, cols, channels, row0, col0, cols if n_cols is None else n_cols, ld_x, ld_out, x_dtype,
                           out_dtype, code, p, seed, offset)


def dropout_add(x, residual=None, p=0.25, seed=0, offset=0, share="none", row0=0, col0=0, n_cols=None, out=None,
                out_dtype=None, stream=None):
    """residual + dropout(x): [rows][cols][channels] float32 or bfloat16 tensors (x and residual of a type each; rows may
    be further apart than cols * channels), the result of the residual's type (without one: out_dtype "f32" or "bf16",
    default x's).  share: "none", "rows" (all rows have the same mask) or "columns".  row0, col0, n_cols: the
    place of a tile in a tensor of n_cols columns.  out may be residual or x itself; its rows are as far apart as
    residual's (without an out, rows that are further apart are copied first)."""
    ld_x = _rows("x", x)
    dt = residual.dtype if residual is not None else x.dtype if out_dtype is None else _t.TORCH_DTYPE[DTYPE_CODE[out_dtype]]
    with on_stream(x.device, stream) as s:
        ld_res = None if residual is None else _rows("residual", residual, x.shape, x.device)
        if out is None:
            ld = x.shape[1] * x.shape[2]
            if ld_res is None or ld_res == ld:
                out = x.new_empty(x.shape, dtype=dt)
            else:                                    # (the kernel has one row stride for both)
                out = residual = residual.contiguous()
        else:
            ld = _rows("out", out, x.shape, x.device)
            if out.dtype != dt:
                raise ValueError(f"out must be {dt}, not {out.dtype}")
            if ld_res is not None and ld_res != ld:
                raise ValueError("residual and out must have the same row stride")
        v = _view(x.shape, ld_x, ld, _DTYPES[x.dtype], _DTYPES[dt], p, seed, offset, share, row0, col0, n_cols)
        pair_dropout_add(v, x, residual, out, s)
    return out


def dropout_backward(dout, p=0.25, seed=0, offset=0, share="none", row0=0, col0=0, n_cols=None, dtype=None, out=None,
                     stream=None):
    """The gradient of x, of type `dtype` ("f32" or "bf16", default dout's), from dout and the arguments of
    dropout_add (the residual's is dout itself).  out may be dout itself."""
    ld_out = _rows("dout", dout)
    dt = dout.dtype if dtype is None else _t.TORCH_DTYPE[DTYPE_CODE[dtype]]
    with on_stream(dout.device, stream) as s:
        dx = dout.new_empty(dout.shape, dtype=dt) if out is None else out
        ld_x = _rows("out", dx, dout.shape, dout.device)
        if dx.dtype != dt:
            raise ValueError(f"out must be {dt}, not {dx.dtype}")
        v = _view(dout.shape, ld_x, ld_out, _DTYPES[dt], _DTYPES[dout.dtype], p, seed, offset, share, row0, col0, n_cols)
        pair_dropout_backward(v, dout, dx, s)
    return dx
