"""Norms of queries and keys for each head with the position rotation in the same pass (include/norm_rotate.h): the C
names, and norm_rotate / norm_rotate_backward, which check their tensors and allocate outputs and workspaces with torch.
Streams and devices as in attention.py."""
import ctypes

import torch

from . import attention as _a
from . import checkpoint8 as _c8
from . import trimul as _t
from .attention import CrossAttnTensor
from .trimul import TRI_MUL_BF16, TRI_MUL_F32, _check, _i32, _i64, _ptr, _vp, on_stream

_DTYPES = {torch.float32: TRI_MUL_F32, torch.bfloat16: TRI_MUL_BF16}
NORMS = {"rms": 0, "layer": 1}
PAIRS = {"halves": 0, "adjacent": 1}


class NormRotateView(ctypes.Structure):
    """norm_rotate_view_t."""
    _fields_ = [("batch", _i64), ("n", _i64), ("d", _i32), ("rot", _i32), ("dtype", _i32), ("weight_dtype", _i32),
                ("layer", _i32), ("adjacent", _i32), ("eps", ctypes.c_float), ("positions", _vp), ("positions_batch", _i64),
                ("freqs", _vp)]


class NormRotateSide(ctypes.Structure):
    """norm_rotate_side_t."""
    _fields_ = [("heads", _i32), ("x", CrossAttnTensor), ("gain", _vp), ("shift", _vp), ("codes", _vp), ("powers", _vp)]


class NormRotateGrad(ctypes.Structure):
    """norm_rotate_grad_t."""
    _fields_ = [("dy", CrossAttnTensor), ("dx", CrossAttnTensor), ("dgain", _vp), ("dshift", _vp)]


_view, _side, _grad = (ctypes.POINTER(t) for t in (NormRotateView, NormRotateSide, NormRotateGrad))
_tensor = ctypes.POINTER(CrossAttnTensor)

# name -> (restype, argtypes); the same order and meaning as include/norm_rotate.h
SIGNATURES = {
    "norm_rotate_forward": (ctypes.c_int, [_view, _side, _side, _tensor, _tensor, _vp]),
    "norm_rotate_backward_workspace_size": (ctypes.c_int, [_view, _side, _side, ctypes.POINTER(ctypes.c_size_t)]),
    "norm_rotate_backward": (ctypes.c_int, [_view, _side, _side, _grad, _grad, _vp, ctypes.c_size_t, _vp]),
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


def norm_rotate_backward_workspace_size(view, q, k):
    n = ctypes.c_size_t()
    _check(lib().norm_rotate_backward_workspace_size(view, q, k, n))
    return n.value


def frequencies(rot, base=10000.0, device="cuda"):
    """base^(-2 i / rot) radians per position for the rot / 2 pairs, float64: what norm_rotate takes as freqs."""
    return torch.tensor([base ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64).to(device)


def _checked(name, t, dtype, device, shape):
    """cross_attn_tensor_t of t after checking type, device, shape and contiguous channels."""
    if t.dtype != dtype or t.device != device or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} {list(shape)} tensor on {device}, not {t.dtype} {list(t.shape)} on {t.device}")
    s = t.stride()
    if s[3] != 1 and shape[3] > 1 and t.numel():
        raise ValueError(f"{name} must have unit stride along its last axis")
    return CrossAttnTensor(t.data_ptr(), s[0], s[1], s[2])


def _call(sides, positions, freqs, norm, pairs, eps):
    """The call's view and its sides; sides: (name, x or Checkpoint8 or None, gain, shift) of the queries and the keys."""
    if norm not in NORMS or pairs not in PAIRS:
        raise ValueError(f"norm must be one of {sorted(NORMS)} and pairs one of {sorted(PAIRS)}, not {norm!r} and {pairs!r}")
    first = next((s[1] for s in sides if s[1] is not None), None)
    if first is None:
        raise ValueError("neither queries nor keys")
    if len(first.shape) != 4:
        raise ValueError("q and k must be [batch][n][heads][d]")
    dtype, device = first.dtype, first.device
    if dtype not in _DTYPES:
        raise ValueError(f"q and k must be float32 or bfloat16, not {dtype}")
    if device.type != "cuda":
        raise ValueError("tensors passed to the library must live on the GPU")
    batch, n, _, d = first.shape
    w = NormRotateView(batch, n, d, 0, _DTYPES[dtype], TRI_MUL_F32, NORMS[norm], PAIRS[pairs], eps)
    if freqs is not None:
        if freqs.dtype != torch.float64 or freqs.device != device or freqs.dim() != 1 or not freqs.is_contiguous():
            raise ValueError(f"freqs must be contiguous float64 [rot / 2] on {device}, not {freqs.dtype} {list(freqs.shape)} on {freqs.device}")
        w.rot, w.freqs = 2 * freqs.numel(), freqs.data_ptr()
    if w.rot:
        if positions is None or positions.dtype != torch.int32 or positions.device != device:
            raise ValueError(f"positions must be an int32 tensor on {device}")
        shape = positions.shape
        if len(shape) not in (1, 2) or shape[-1] != n or (len(shape) == 2 and shape[0] not in (1, batch)) or (n > 1 and positions.stride(-1) != 1):
            raise ValueError(f"positions must be [{n}] or [{batch} or 1][{n}] with unit stride, not {list(shape)}")
        w.positions = positions.data_ptr()
        w.positions_batch = positions.stride(0) if len(shape) == 2 and shape[0] > 1 else 0
    weight, held = None, isinstance(first, _c8.Checkpoint8)
    result = []
    for name, x, gain, shift in sides:
        if x is None:
            if gain is not None or shift is not None:
                raise ValueError(f"weights of {name}, which is missing")
            result.append(None)
            continue
        shape = x.shape
        if len(shape) != 4:
            raise ValueError("q and k must be [batch][n][heads][d]")
        heads = shape[2]
        if isinstance(x, _c8.Checkpoint8) != held:
            raise ValueError("q and k are both tensors or both checkpoints")
        addresses = []
        for what, t in (("gain", gain), ("shift", shift)):
            if t is None:
                addresses.append(None)
                continue
            if t.dtype not in _DTYPES or t.device != device or t.shape != (d,) or not t.is_contiguous():
                raise ValueError(f"{what} of {name} must be contiguous float32 or bfloat16 [{d}] on {device}, not {t.dtype} {list(t.shape)} on {t.device}")
            if weight is not None and t.dtype != weight:
                raise ValueError("gains and shifts must be of one type")
            weight = t.dtype
            addresses.append(t.data_ptr())
        if held:
            if shape != (batch, n, heads, d) or x.dtype != dtype or x.device != device or x.group != d:
                raise ValueError(f"{name} must be a checkpoint of a {dtype} {[batch, n, heads, d]} tensor on {device} in groups of {d}")
            result.append(NormRotateSide(heads, CrossAttnTensor(), *addresses, x.codes.data_ptr(), x.powers.data_ptr()))
        else:
            result.append(NormRotateSide(heads, _checked(name, x, dtype, device, (batch, n, heads, d)), *addresses))
    if weight is not None:
        w.weight_dtype = _DTYPES[weight]
    return w, result


def _dense(t, n, heads, d):
    """cross_attn_tensor_t of a contiguous [batch][n][heads][d] tensor."""
    return CrossAttnTensor(t.data_ptr(), n * heads * d, heads * d, d)


def norm_rotate(q, k, positions=None, freqs=None, gain_q=None, gain_k=None, shift_q=None, shift_k=None, norm="rms",
                pairs="halves", eps=1e-6, checkpoint=False, out_q=None, out_k=None, stream=None):
    """(yq, yk): q and k normalised by head, scaled, and turned by their positions; with checkpoint also the two
    Checkpoint8 of q and k that norm_rotate_backward takes in their place.

    q, k: [batch][n][heads][d] (heads each their own), float32 or bfloat16, strides multiples of 16 bytes (slices of one
    projection are fine); either may be None, and so are its results.  d: a multiple of 8 up to 256.  freqs: float64
    [rot / 2] (frequencies(rot)), rot a multiple of 8 up to d; None: no rotation.  positions: int32 [n] or [batch][n].
    gain, shift: [d], of one type; None: 1 and 0.  norm: "rms" or "layer" (the mean removed).  pairs: "halves" (channel m
    with m + rot / 2) or "adjacent" (2m with 2m + 1).  out_q, out_k may be q and k themselves."""
    w, (sq, sk) = _call((("q", q, gain_q, shift_q), ("k", k, gain_k, shift_k)), positions, freqs, norm, pairs, eps)
    first = q if q is not None else k
    if not isinstance(first, torch.Tensor):
        raise ValueError("q and k must be tensors")
    ys, to, held = [], [], []
    with on_stream(first.device, stream) as s:
        for x, side, out, name in ((q, sq, out_q, "out_q"), (k, sk, out_k, "out_k")):
            if x is None:
                if out is not None:
                    raise ValueError(f"{name} without its input")
                ys.append(None)
                to.append(None)
                held.append(None)
                continue
            shape = x.shape
            if out is None:
                out = x.new_empty(shape)
                to.append(_dense(out, w.n, shape[2], w.d))
            else:
                to.append(_checked(name, out, x.dtype, x.device, shape))
            ys.append(out)
            if checkpoint:
                c = _c8.Checkpoint8(torch.empty(shape, dtype=torch.int8, device=x.device),
                                    torch.empty((w.batch, w.n, shape[2], 1), dtype=torch.uint8, device=x.device), w.d, x.dtype)
                side.codes, side.powers = c.codes.data_ptr(), c.powers.data_ptr()
                held.append(c)
        _check(lib().norm_rotate_forward(w, sq, sk, to[0], to[1], s))
    return tuple(ys + held) if checkpoint else tuple(ys)


def norm_rotate_backward(q, k, dyq, dyk, positions=None, freqs=None, gain_q=None, gain_k=None, shift_q=None, shift_k=None,
                         norm="rms", pairs="halves", eps=1e-6, stream=None):
    """(dq, dk, grads) for dyq and dyk from the forward's arguments; q and k may be the forward's Checkpoint8.  grads:
    gain_q, gain_k, shift_q, shift_k as float32 [d] (None where there is no such weight)."""
    w, (sq, sk) = _call((("q", q, gain_q, shift_q), ("k", k, gain_k, shift_k)), positions, freqs, norm, pairs, eps)
    first = q if q is not None else k
    weights = {"gain_q": gain_q, "gain_k": gain_k, "shift_q": shift_q, "shift_k": shift_k}
    there = [name for name, t in weights.items() if t is not None]
    with on_stream(first.device, stream) as s:
        grads = dict.fromkeys(weights)
        if there:                                   # (one allocation for all of them)
            grads.update(zip(there, torch.empty((len(there), w.d), dtype=torch.float32, device=first.device).unbind()))
        dxs, gs = [], []
        for x, dy, name in ((q, dyq, "q"), (k, dyk, "k")):
            if (x is None) != (dy is None):
                raise ValueError(f"{name} and dy{name} are both given or both None")
            if x is None:
                dxs.append(None)
                gs.append(None)
                continue
            shape = x.shape
            td = _checked("dy" + name, dy, x.dtype, x.device, shape)
            dx = torch.empty(shape, dtype=x.dtype, device=x.device)
            dxs.append(dx)
            gs.append(NormRotateGrad(td, _dense(dx, w.n, shape[2], w.d), _ptr(grads["gain_" + name]), _ptr(grads["shift_" + name])))
        n = norm_rotate_backward_workspace_size(w, sq, sk)
        ws = torch.empty(n, dtype=torch.uint8, device=first.device) if n else None
        _check(lib().norm_rotate_backward(w, sq, sk, gs[0], gs[1], _ptr(ws), n, s))
    return dxs[0], dxs[1], grads
