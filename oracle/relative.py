"""fp64 CPU oracle for the relative position bias by buckets.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import or call
this module.  It shares no code with the HIP library.
"""
import numpy as np

from .trimul import f64


def buckets(lut, rows, pos_q, pos_k, seg_q=None, seg_k=None):
    """Row of the table for each (query, key): lut of the distance key - query cut off at its ends, the last row where
    the segments differ."""
    reach = len(lut) // 2
    far = np.asarray(pos_k, dtype=np.int64)[None, :] - np.asarray(pos_q, dtype=np.int64)[:, None]
    b = np.asarray(lut)[np.clip(far, -reach, reach) + reach]
    if seg_q is not None:
        b = np.where(np.asarray(seg_q)[:, None] == np.asarray(seg_k)[None, :], b, rows - 1)
    return b


def relative_bias(table, b, base=None):
    """[heads][nq][nk]"""
    out = np.moveaxis(f64(table)[b], -1, 0)
    return out if base is None else f64(base) + out


def relative_pair(table, b, base=None):
    """[nq][nk][channels]"""
    return f64(table)[b] if base is None else f64(base) + f64(table)[b]


def table_gradient(dout, b, rows):
    """[rows][channels] from dout [nq][nk][channels]."""
    d = f64(dout)
    return np.stack([d[b == t].sum(axis=0) for t in range(rows)])


def log_bucket(distance, single, steps, reach):
    """Bucket of a distance >= 0 by its logarithm, `single` single distances and then `steps` steps up to `reach`: exact,
    by comparing whole powers."""
    if distance < single:
        return distance
    return single + max(k for k in range(steps) if distance ** steps * single ** k >= reach ** k * single ** steps)
