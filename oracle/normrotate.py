"""fp64 CPU oracle for the norms of queries and keys by head with the position rotation, and their gradients.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import or call
this module.  It shares no code with the HIP library.
"""
import numpy as np

from .trimul import f64


def _turned(x, phase, pairs):
    """The first channels of x [..., n, heads, d] as complex numbers, times phase [..., n, rot / 2]."""
    half = phase.shape[-1]
    y = x.copy()
    if pairs == "halves":
        z = (x[..., :half] + 1j * x[..., half:2 * half]) * phase[..., None, :]
        y[..., :half], y[..., half:2 * half] = z.real, z.imag
    else:
        z = (x[..., 0:2 * half:2] + 1j * x[..., 1:2 * half:2]) * phase[..., None, :]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = z.real, z.imag
    return y


def phases(positions, freqs):
    """exp(i p f), [..., n, rot / 2]."""
    return np.exp(1j * np.asarray(positions, dtype=np.float64)[..., None] * f64(freqs))


def normalise(x, norm, eps):
    """(u, r) of rows along the last axis."""
    x = f64(x)
    if norm == "layer":
        x = x - x.mean(axis=-1, keepdims=True)
    r = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return x * r, r


def norm_rotate(x, phase, gain=None, shift=None, norm="rms", pairs="halves", eps=1e-6):
    w = normalise(x, norm, eps)[0]
    w = w if gain is None else w * f64(gain)
    return _turned(w if shift is None else w + f64(shift), phase, pairs)


def norm_rotate_backward(x, dy, phase, gain=None, norm="rms", pairs="halves", eps=1e-6):
    """(dx, dgain, dshift)"""
    u, r = normalise(x, norm, eps)
    g = _turned(f64(dy), phase.conj(), pairs)
    rows = tuple(range(g.ndim - 1))
    h = g if gain is None else g * f64(gain)
    dx = h - u * (h * u).mean(axis=-1, keepdims=True)
    if norm == "layer":
        dx = dx - h.mean(axis=-1, keepdims=True)
    return dx * r, (g * u).sum(axis=rows), g.sum(axis=rows)
