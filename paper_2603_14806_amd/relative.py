"""Learned relative position bias by buckets (include/relative_bias.h): the C names; Buckets, which says which distance
has which row of the table; relative_bias, the bias that attention.cross_attention takes, and relative_pair, the relative
position encoding of a pair tensor, each with the gradient of the table.  Streams and devices as in attention.py."""
import ctypes

import torch

from . import attention as _a
from . import trimul as _t
from .attention import CrossAttnBias, bias_tensor
from .trimul import DTYPE_CODE, TORCH_DTYPE, TRI_MUL_BF16, TRI_MUL_F32, _check, _i32, _i64, _ptr, _vp, on_stream

_DTYPES = {torch.float32: TRI_MUL_F32, torch.bfloat16: TRI_MUL_BF16}


class RelativeView(ctypes.Structure):
    """relative_view_t."""
    _fields_ = [("batch", _i64), ("nq", _i64), ("nk", _i64), ("heads", _i32), ("dtype", _i32), ("table_dtype", _i32),
                ("buckets", _i32), ("reach", _i32), ("lut", _vp), ("pos_q", _vp), ("pos_k", _vp), ("pos_q_batch", _i64),
                ("pos_k_batch", _i64), ("seg_q", _vp), ("seg_k", _vp), ("seg_q_batch", _i64), ("seg_k_batch", _i64)]


_view, _bias, _size = ctypes.POINTER(RelativeView), ctypes.POINTER(CrossAttnBias), ctypes.POINTER(ctypes.c_size_t)

# name -> (restype, argtypes); the same order and meaning as include/relative_bias.h
SIGNATURES = {
    "relative_bias": (ctypes.c_int, [_view, _vp, _bias, _bias, _vp]),
    "relative_bias_backward_workspace_size": (ctypes.c_int, [_view, _size]),
    "relative_bias_backward": (ctypes.c_int, [_view, _bias, _vp, _vp, ctypes.c_size_t, _vp]),
    "relative_pair": (ctypes.c_int, [_view, _vp, _vp, _i64, _vp, _i64, _vp]),
    "relative_pair_backward_workspace_size": (ctypes.c_int, [_view, _size]),
    "relative_pair_backward": (ctypes.c_int, [_view, _vp, _i64, _vp, _vp, ctypes.c_size_t, _vp]),
}

_lib = None


def lib():
    """libtrimul.so with this module's signatures set."""
    global _lib
    if _lib is None:
        L = _a.lib()
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


# ---------------------------------------------------------------- C names (the others' names are those of the torch calls below)

def relative_bias_backward_workspace_size(view):
    n = ctypes.c_size_t()
    _check(lib().relative_bias_backward_workspace_size(view, n))
    return n.value


def relative_pair_backward_workspace_size(view):
    n = ctypes.c_size_t()
    _check(lib().relative_pair_backward_workspace_size(view, n))
    return n.value


# ---------------------------------------------------------------- buckets

class Buckets:
    """The row of the table for each distance key - query in [-reach, reach] (beyond it: the row of its end), held on one
    GPU; `rows` is the number of rows of the table.  With `other` the table has one more row, for the pairs whose query
    and key are of different segments (chains)."""

    def __init__(self, lut, other=False, device="cuda"):
        lut = [int(b) for b in lut]
        if len(lut) % 2 != 1 or len(lut) > 2 * 4095 + 1:
            raise ValueError(f"lut must have 2 reach + 1 entries, reach at most 4095, not {len(lut)}")
        if min(lut) < 0 or max(lut) + 1 + bool(other) > 256:
            raise ValueError("buckets must be in [0, 256), the one for other segments included")
        self.reach, self.other = len(lut) // 2, bool(other)
        self.rows = max(lut) + 1 + self.other
        self.lut = torch.tensor(lut, dtype=torch.uint8).to(device)

    @classmethod
    def clipped(cls, reach, other=False, device="cuda"):
        """A bucket for each distance, 2 reach + 1 of them."""
        return cls(range(2 * reach + 1), other, device)

    @classmethod
    def logarithmic(cls, buckets, reach, both=True, other=False, device="cuda"):
        """`buckets` rows: of the keys before the query (both: half of the rows, and the other half for the keys behind
        it), the first half single distances, the others evenly spaced in the logarithm up to `reach`, where the last
        one starts or has started.  Without both, keys behind the query are in bucket 0.  The borders are found in whole
        numbers: distance r is in step k or a later one where (r / m)^K >= (reach / m)^k, for m single distances and K steps."""
        per = buckets // 2 if both else buckets
        single = per // 2
        steps = per - single
        if single < 1 or (both and buckets % 2) or reach <= single:
            raise ValueError(f"{buckets} buckets up to a reach of {reach}: single distances, and a reach beyond them, are needed")
        past, k = [], 0
        for r in range(reach + 1):
            while r >= single and k + 1 < steps and r ** steps >= reach ** (k + 1) * single ** (steps - k - 1):
                k += 1
            past.append(r if r < single else single + k)
        ahead = [per + b if both else 0 for b in past]
        return cls(past[:0:-1] + [past[0]] + ahead[1:], other, device)


# ---------------------------------------------------------------- torch tensors

def _places(name, t, n, device):
    """(address, entries, stride from one entry to the next) of [n] or [entries][n] int32 values."""
    if t.dtype != torch.int32 or t.device != device:
        raise ValueError(f"{name} must be an int32 tensor on {device}, not {t.dtype} on {t.device}")
    if t.dim() not in (1, 2) or (n is not None and t.shape[-1] != n) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be [{'n' if n is None else n}] or [entries][{'n' if n is None else n}] with unit stride, not {list(t.shape)}")
    entries = t.shape[0] if t.dim() == 2 else 1
    return t.data_ptr(), entries, t.stride(0) if entries > 1 else 0


def _call(device, dtype, heads, buckets, pos_q, pos_k, seg_q, seg_k, batch, nq=None, nk=None, table=None):
    """The call's relative_view_t; batch None: what the positions say."""
    if not isinstance(buckets, Buckets):
        raise ValueError("buckets must be a relative.Buckets")
    if device.type != "cuda":
        raise ValueError("tensors passed to the library must live on the GPU")
    if buckets.lut.device != device:
        raise ValueError(f"buckets must live on {device}, not on {buckets.lut.device}")
    if dtype not in _DTYPES:
        raise ValueError(f"the bias must be float32 or bfloat16, not {dtype}")
    w = RelativeView(0, 0, 0, heads, _DTYPES[dtype], TRI_MUL_F32, buckets.rows, buckets.reach, buckets.lut.data_ptr())
    if table is not None:
        if table.dtype not in _DTYPES or table.device != device or table.shape != (buckets.rows, heads) or not table.is_contiguous():
            raise ValueError(f"table must be a contiguous float32 or bfloat16 [{buckets.rows}][{heads}] tensor on {device}, not {table.dtype} {list(table.shape)} on {table.device}")
        w.table_dtype = _DTYPES[table.dtype]
    if (seg_q is None) != (seg_k is None):
        raise ValueError("segments of the queries and the keys are both given or both None")
    if seg_q is not None and not buckets.other:
        raise ValueError("segments need buckets with a row for other segments (other=True)")
    w.pos_q, eq, w.pos_q_batch = _places("pos_q", pos_q, nq, device)
    w.pos_k, ek, w.pos_k_batch = _places("pos_k", pos_k, nk, device)
    w.nq, w.nk = pos_q.shape[-1], pos_k.shape[-1]
    entries = {eq, ek}
    if seg_q is not None:
        w.seg_q, e, w.seg_q_batch = _places("seg_q", seg_q, w.nq, device)
        w.seg_k, f, w.seg_k_batch = _places("seg_k", seg_k, w.nk, device)
        entries |= {e, f}
        if not w.nq or not w.nk:
            w.seg_q = w.seg_k = None
    entries.discard(1)
    if len(entries) > 1 or (batch is not None and batch != 1 and entries - {batch}) or (batch == 1 and entries):
        raise ValueError(f"positions and segments are of {sorted(entries)} entries" + (f", not {batch}" if batch is not None else ""))
    w.batch = batch if batch is not None else entries.pop() if entries else 1
    return w


def _bias_strides(name, t, w, dtype, whole):
    """cross_attn_bias_t of a [batch][heads][nq][nk] tensor (not whole: an axis of length 1 repeats it)."""
    n, s = t.shape, t.stride()
    if t.dtype != dtype or len(n) != 4 or n[2] != w.nq or n[3] != w.nk or n[0] not in (w.batch, w.batch if whole else 1) or n[1] not in (w.heads, w.heads if whole else 1):
        one = "" if whole else " or 1"
        raise ValueError(f"{name} must be a {dtype} [{w.batch}{one}][{w.heads}{one}][{w.nq}][{w.nk}] tensor, not {t.dtype} {list(n)}")
    if w.nk > 1 and s[3] != 1 and t.numel():
        raise ValueError(f"{name} must have unit stride along its last axis")
    return bias_tensor(t)


def _four(t):
    return t if t is None or t.dim() != 3 else t[None]


def relative_bias(table, buckets, pos_q, pos_k, seg_q=None, seg_k=None, base=None, out=None, dtype=None, stream=None):
    """out [batch][heads][nq][nk] = base + table[bucket], of type `dtype` ("f32" or "bf16"; default base's, else the
    table's), its rows padded to a multiple of 8 values as cross_attention takes them.

    table: [buckets.rows][heads], float32 or bfloat16.  pos_q, pos_k (and seg_q, seg_k): int32, [n] or [batch][n].  base:
    [batch or 1][heads or 1][nq][nk] (or without the first axis), an axis of length 1 is shared.  batch is the largest of
    these.  out may be base itself; without one the padding behind nk is unspecified."""
    base, device = _four(base), table.device
    if table.dim() != 2:
        raise ValueError(f"table must be [{getattr(buckets, 'rows', 'rows')}][heads], not {list(table.shape)}")
    dt = TORCH_DTYPE[DTYPE_CODE[dtype]] if dtype is not None else base.dtype if base is not None else table.dtype
    if base is not None and base.device != device:
        raise ValueError(f"base must live on {device}, not on {base.device}")
    batch = base.shape[0] if base is not None and base.dim() == 4 and base.shape[0] != 1 else None
    w = _call(device, dt, table.shape[1], buckets, pos_q, pos_k, seg_q, seg_k, batch, table=table)
    tb = None if base is None else _bias_strides("base", base, w, dt, False)
    with on_stream(device, stream) as s:
        shape = (w.batch, w.heads, w.nq, w.nk)
        if out is None:
            out = torch.empty(shape[:3] + (-(-w.nk // 8) * 8,), dtype=dt, device=device)[..., :w.nk]
        elif out.device != device:
            raise ValueError(f"out must live on {device}, not on {out.device}")
        to = _bias_strides("out", _four(out), w, dt, True)
        _check(lib().relative_bias(w, table.data_ptr(), tb, to, s))
    return out


def relative_bias_backward(dout, buckets, pos_q, pos_k, seg_q=None, seg_k=None, stream=None):
    """The gradient of the table, [buckets.rows][heads] float32, from dout [batch][heads][nq][nk] (or without the first
    axis) of a relative_bias of these arguments -- cross_attention_backward's dbias as it comes.  (base's is dout, summed
    over the axes that it shares.)"""
    dout = _four(dout)
    if dout.dim() != 4:
        raise ValueError(f"dout must be [batch][heads][nq][nk], not {list(dout.shape)}")
    batch, heads, nq, nk = dout.shape
    w = _call(dout.device, dout.dtype, heads, buckets, pos_q, pos_k, seg_q, seg_k, batch, nq, nk)
    td = _bias_strides("dout", dout, w, dout.dtype, True)
    with on_stream(dout.device, stream) as s:
        dtable = torch.empty((buckets.rows, heads), dtype=torch.float32, device=dout.device)
        n = relative_bias_backward_workspace_size(w)
        ws = torch.empty(n, dtype=torch.uint8, device=dout.device) if n else None
        _check(lib().relative_bias_backward(w, td, dtable.data_ptr(), _ptr(ws), n, s))
    return dtable


def _rows(name, t, w, dtype, device):
    """Elements from one row to the next of a [nq][nk][channels] tensor whose rows are contiguous."""
    if t.dtype != dtype or t.device != device or t.shape != (w.nq, w.nk, w.heads):
        raise ValueError(f"{name} must be a {dtype} [{w.nq}][{w.nk}][{w.heads}] tensor on {device}, not {t.dtype} {list(t.shape)} on {t.device}")
    sr, sc, sch = t.stride()
    if t.numel() and ((w.heads > 1 and sch != 1) or (w.nk > 1 and sc != w.heads)):
        raise ValueError(f"{name}'s columns and channels must be contiguous")
    return sr if w.nq > 1 else w.nk * w.heads


def relative_pair(table, buckets, pos_q, pos_k, seg_q=None, seg_k=None, base=None, out=None, dtype=None, stream=None):
    """out [rows][cols][channels] = base + table[bucket]: the relative position encoding added to the pair tensor base (its
    rows may be further apart than cols * channels), of base's type (without one: `dtype`, default the table's).  The rows
    are at pos_q (and of segments seg_q), the columns at pos_k: a tile of a 2-D grid passes its own.  out may be base."""
    device = table.device
    if table.dim() != 2:
        raise ValueError(f"table must be [{getattr(buckets, 'rows', 'rows')}][channels], not {list(table.shape)}")
    dt = TORCH_DTYPE[DTYPE_CODE[dtype]] if dtype is not None else base.dtype if base is not None else table.dtype
    w = _call(device, dt, table.shape[1], buckets, pos_q, pos_k, seg_q, seg_k, 1, table=table)
    ld_base = 0 if base is None else _rows("base", base, w, dt, device)
    with on_stream(device, stream) as s:
        if out is None:
            out = torch.empty((w.nq, w.nk, w.heads), dtype=dt, device=device)
        ld = _rows("out", out, w, dt, device)
        _check(lib().relative_pair(w, table.data_ptr(), _ptr(base), ld_base, out.data_ptr(), ld, s))
    return out


def relative_pair_backward(dout, buckets, pos_q, pos_k, seg_q=None, seg_k=None, stream=None):
    """The gradient of the table, [buckets.rows][channels] float32, from dout [rows][cols][channels] of a relative_pair of
    these arguments (base's is dout itself)."""
    if dout.dim() != 3:
        raise ValueError(f"dout must be [rows][cols][channels], not {list(dout.shape)}")
    w = _call(dout.device, dout.dtype, dout.shape[2], buckets, pos_q, pos_k, seg_q, seg_k, 1, dout.shape[0], dout.shape[1])
    ld = _rows("dout", dout, w, dout.dtype, dout.device)
    with on_stream(dout.device, stream) as s:
        dtable = torch.empty((buckets.rows, w.heads), dtype=torch.float32, device=dout.device)
        n = relative_pair_backward_workspace_size(w)
        ws = torch.empty(n, dtype=torch.uint8, device=dout.device) if n else None
        _check(lib().relative_pair_backward(w, dout.data_ptr(), ld, dtable.data_ptr(), _ptr(ws), n, s))
    return dtable
