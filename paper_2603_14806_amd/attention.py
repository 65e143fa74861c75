"""Attention of queries over keys of another length (include/cross_attn.h):
the C names, and cross_attention / cross_attention_backward, which check their
tensors and allocate outputs and workspaces with torch.

Every call runs on the device its tensors are on, on `stream` (a torch stream
or a raw hipStream_t) or that device's current stream, and allocates there.
"""
import ctypes

import torch

from . import trimul as _t
from .trimul import TRI_MUL_BF16, TRI_MUL_F32, _check, _i32, _i64, _ptr, _vp, on_stream

_DTYPES = {torch.float32: TRI_MUL_F32, torch.bfloat16: TRI_MUL_BF16}


class CrossAttnTensor(ctypes.Structure):
    """cross_attn_tensor_t."""
    _fields_ = [("data", _vp), ("batch", _i64), ("token", _i64), ("head", _i64)]


class CrossAttnBias(ctypes.Structure):
    """cross_attn_bias_t."""
    _fields_ = [("data", _vp), ("batch", _i64), ("head", _i64), ("row", _i64)]


class CrossAttnView(ctypes.Structure):
    """cross_attn_view_t."""
    _fields_ = [("batch", _i64), ("nq", _i64), ("nk", _i64), ("heads", _i32), ("kv_heads", _i32), ("d", _i32),
                ("dtype", _i32), ("scale", ctypes.c_float), ("bias", CrossAttnBias), ("mask", _vp), ("mask_batch", _i64)]


_view, _tensor, _size = ctypes.POINTER(CrossAttnView), ctypes.POINTER(CrossAttnTensor), ctypes.POINTER(ctypes.c_size_t)

# name -> (restype, argtypes); the same order and meaning as include/cross_attn.h
SIGNATURES = {
    "cross_attn_workspace_size": (ctypes.c_int, [_view, _size]),
    "cross_attn_stats_size": (ctypes.c_int, [_view, _size]),
    "cross_attn_forward": (ctypes.c_int, [_view, _tensor, _tensor, _tensor, _tensor, _vp, _vp, ctypes.c_size_t, _vp]),
    "cross_attn_backward_workspace_size": (ctypes.c_int, [_view, _size]),
    "cross_attn_backward": (ctypes.c_int, [_view] + [_tensor] * 4 + [_vp] + [_tensor] * 4 +
                            [ctypes.POINTER(CrossAttnBias), _vp, ctypes.c_size_t, _vp]),
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


# ---------------------------------------------------------------- C names
#
# Structures are passed as they are (ctypes takes their address), pointers as tensors or addresses.

def cross_attn_workspace_size(view):
    n = ctypes.c_size_t()
    _check(lib().cross_attn_workspace_size(view, n))
    return n.value


def cross_attn_stats_size(view):
    n = ctypes.c_size_t()
    _check(lib().cross_attn_stats_size(view, n))
    return n.value


def cross_attn_forward(view, q, k, v, out, stats, ws, ws_bytes, stream=None):
    _check(lib().cross_attn_forward(view, q, k, v, out, _ptr(stats), _ptr(ws), ws_bytes, _t._stream(stream)))


def cross_attn_backward_workspace_size(view):
    n = ctypes.c_size_t()
    _check(lib().cross_attn_backward_workspace_size(view, n))
    return n.value


def cross_attn_backward(view, q, k, v, out, stats, dout, dq, dk, dv, dbias, ws, ws_bytes, stream=None):
    _check(lib().cross_attn_backward(view, q, k, v, out, _ptr(stats), dout, dq, dk, dv, dbias, _ptr(ws), ws_bytes,
                                     _t._stream(stream)))


# ---------------------------------------------------------------- torch tensors

def tensor(t):
    """cross_attn_tensor_t of a [batch][tokens][heads][d] GPU tensor (kept alive by the caller)."""
    s = t.stride()
    return CrossAttnTensor(t.data_ptr(), s[0], s[1], s[2])


def bias_tensor(t):
    """cross_attn_bias_t of a [batch or 1][heads or 1][nq][nk] GPU tensor: an axis of length 1 is shared."""
    n, s = t.shape, t.stride()
    return CrossAttnBias(t.data_ptr(), 0 if n[0] == 1 else s[0], 0 if n[1] == 1 else s[1], s[2])


def _checked(name, t, dtype, device, shape):
    """tensor(t) after checking that t has this type, device and shape, and contiguous channels."""
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor on {device}, not {t.dtype} on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    s = t.stride()
    if s[3] != 1 and shape[3] > 1:
        raise ValueError(f"{name} must have unit stride along its last axis")
    return CrossAttnTensor(t.data_ptr(), s[0], s[1], s[2])


def _checked_bias(t, batch, heads, nq, nk):
    """bias_tensor(t) after checking its shape, unit stride along the keys, and that the padding of its last row, which
    is read up to a multiple of 8 values, is memory of t's."""
    if t.dim() == 3:
        t = t[None]
    n = t.shape
    if len(n) != 4 or n[0] not in (1, batch) or n[1] not in (1, heads) or n[2] != nq or n[3] != nk:
        raise ValueError(f"bias must be [{batch} or 1][{heads} or 1][{nq}][{nk}], not {list(n)}")
    if not t.numel():
        return CrossAttnBias()
    s = t.stride()
    if nk > 1 and s[3] != 1:
        raise ValueError("bias must have unit stride along its last axis")
    end = t.storage_offset() + (n[0] - 1) * s[0] + (n[1] - 1) * s[1] + (nq - 1) * s[2] + (nk + 7) // 8 * 8
    if (nq == 1 or s[2] % 8 == 0) and end * t.element_size() > t.untyped_storage().nbytes():
        raise ValueError("bias must be a view of a padded tensor: its last row is read up to a multiple of 8 values, past the end of its memory")
    return bias_tensor(t)


def view(q, k, v, bias=None, mask=None, scale=None):
    """cross_attn_view_t of the call (the tensors are kept alive by the caller), after checking shapes and types."""
    return _call(q, k, v, bias, mask, scale)[0]


def _call(q, k, v, bias, mask, scale):
    """The call's cross_attn_view_t and its q, k and v."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v must be [batch][tokens][heads][d]")
    dtype, shape = q.dtype, q.shape
    if dtype not in _DTYPES:
        raise ValueError(f"q must be float32 or bfloat16, not {dtype}")
    if not q.is_cuda:
        raise ValueError("tensors passed to the library must live on the GPU")
    device = q.device
    batch, nq, heads, d = shape
    _, nk, kv_heads, _ = k.shape
    keys = (batch, nk, kv_heads, d)
    args = _checked("q", q, dtype, device, shape), _checked("k", k, dtype, device, keys), _checked("v", v, dtype, device, keys)
    w = CrossAttnView(batch, nq, nk, heads, kv_heads, d, _DTYPES[dtype], max(d, 1) ** -0.5 if scale is None else scale)
    if bias is not None:
        if bias.dtype != dtype or bias.device != device:
            raise ValueError(f"bias must be a {dtype} tensor on {device}")
        w.bias = _checked_bias(bias, batch, heads, nq, nk)
    if mask is not None:
        if mask.dtype not in (torch.uint8, torch.bool) or mask.device != device:
            raise ValueError(f"mask must be a uint8 or bool tensor on {device}")
        if mask.dim() == 1:
            mask = mask[None]
        if mask.dim() != 2 or mask.shape[0] not in (1, batch) or mask.shape[1] != nk or (nk > 1 and mask.stride(1) != 1):
            raise ValueError(f"mask must be [{batch} or 1][{nk}] with unit stride along the keys")
        if mask.numel():
            w.mask = mask.data_ptr()
            w.mask_batch = 0 if mask.shape[0] == 1 else mask.stride(0)
    return (w,) + args


def cross_attention(q, k, v, bias=None, mask=None, scale=None, return_stats=False, stream=None):
    """out [batch][nq][heads][d] of q's type from q and k, v [batch][nk][kv_heads][d] (float32 or bfloat16; heads a
    multiple of kv_heads, d a multiple of 8 up to 128; any strides that are multiples of 16 bytes).

    bias: [batch or 1][heads or 1][nq][nk] (or without the first axis) of q's type whose rows are a multiple of 8
    values apart (a view of a padded tensor is fine; rows are read up to a multiple of 8 values, a single query's
    too); an axis of length 1 is shared.  -inf gives a key weight 0 for one query, but its k and v are multiplied all
    the same: NaN or infinities there show.  mask: [batch or 1][nk] or [nk], uint8 or bool, nonzero where the key is
    present (an absent key's k, v and bias may hold anything).  scale: default 1 / sqrt(d).  With return_stats also
    what cross_attention_backward takes: a flat float32 tensor of the library's own layout (first the maxima and the
    sums, [2][batch][heads][nq])."""
    w, tq, tk, tv = _call(q, k, v, bias, mask, scale)
    with on_stream(q.device, stream) as s:
        out = q.new_empty(q.shape)
        stats = torch.empty(-(-cross_attn_stats_size(w) // 4), dtype=torch.float32, device=q.device) if return_stats else None
        n = cross_attn_workspace_size(w)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        cross_attn_forward(w, tq, tk, tv, tensor(out), stats, ws, n, s)
    return (out, stats) if return_stats else out


def cross_attention_backward(q, k, v, out, stats, dout, bias=None, mask=None, scale=None, need_kv=True,
                             need_bias=True, stream=None):
    """(dq, dk, dv, dbias) for dout, from the forward's arguments, its out and its stats.  dk and dv are None
    without need_kv, dbias is None without a bias or need_bias; dbias has the bias's shape, its rows padded to a
    multiple of 8 values as the bias's are (the view returned ends at nk)."""
    w, tq, tk, tv = _call(q, k, v, bias, mask, scale)
    if need_bias and bias is not None and any(n > 1 and st == 0 for n, st in zip(bias.shape[:-1], bias.stride())):
        raise ValueError("a bias that is repeated along an axis has that axis of length 1 for its gradient")
    to, tg = (_checked(n, t, q.dtype, q.device, q.shape) for n, t in (("out", out), ("dout", dout)))
    if stats.dtype != torch.float32 or stats.device != q.device or stats.dim() != 1 or not stats.is_contiguous() or 4 * stats.numel() < cross_attn_stats_size(w):
        raise ValueError("stats must be the tensor that the forward of these arguments returned")
    with on_stream(q.device, stream) as s:
        dq = q.new_empty(q.shape)
        dk, dv = (k.new_empty(k.shape), v.new_empty(v.shape)) if need_kv else (None, None)
        dbias, grad = None, None
        if bias is not None and need_bias:
            dbias = torch.empty(tuple(bias.shape[:-1]) + (-(-w.nk // 8) * 8,), dtype=q.dtype, device=q.device)[..., :w.nk]
            if w.bias.data:
                grad = bias_tensor(dbias if dbias.dim() == 4 else dbias[None])
        n = cross_attn_backward_workspace_size(w)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device)
        cross_attn_backward(w, tq, tk, tv, to, stats, tg, tensor(dq),
                            tensor(dk) if need_kv else None, tensor(dv) if need_kv else None, grad, ws, n, s)
    return dq, dk, dv, dbias
