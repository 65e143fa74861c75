"""fp64 CPU oracle for the residual addition with dropout.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import or call
this module.  It shares no code with the HIP library.

Generator: Philox-4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random
numbers: as easy as 1, 2, 3", SC 2011), on Python integers held in uint64
arrays.  keep() is the mask of the tile of a [*][n_cols][channels] tensor that
starts at (row0, col0); dropout_add and dropout_backward apply it.
"""
import numpy as np

from .trimul import f64

MASK = (1 << 32) - 1


def philox(counter, key):
    """Ten rounds: counter [..., 4] and key (k0, k1) of 32-bit words -> [..., 4] words (uint64)."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a = c[0] * np.uint64(0xD2511F53)
        b = c[2] * np.uint64(0xCD9E8D57)
        hi = np.uint64(32)
        lo = np.uint64(MASK)
        c = [(b >> hi) ^ c[1] ^ np.uint64(k[0]), b & lo, (a >> hi) ^ c[3] ^ np.uint64(k[1]), a & lo]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return np.stack(c, -1)


def keep(rows, cols, channels, p, seed, offset, share, row0=0, col0=0, n_cols=None):
    """Boolean [rows][cols][channels]; share "none", "rows" or "columns"."""
    n_cols = cols if n_cols is None else n_cols
    r = np.arange(row0, row0 + rows, dtype=np.uint64)[:, None, None] * np.uint64(0 if share == "rows" else 1)
    s = np.arange(col0, col0 + cols, dtype=np.uint64)[None, :, None] * np.uint64(0 if share == "columns" else 1)
    e = (r * np.uint64(n_cols) + s) * np.uint64(channels) + np.arange(channels, dtype=np.uint64)
    block = e >> np.uint64(2)
    full = np.stack([block & np.uint64(MASK), block >> np.uint64(32), np.full_like(block, offset & MASK),
                     np.full_like(block, offset >> 32)], -1)
    words = philox(full, (seed & MASK, seed >> 32))
    word = np.take_along_axis(words, (e & np.uint64(3)).astype(np.int64)[..., None], -1)[..., 0]
    return word >= np.uint64(round(p * 2 ** 32))


def dropout_add(x, res, p, mask):
    return (0.0 if res is None else f64(res)) + np.where(mask, f64(x) / (1 - p), 0.0)


def dropout_backward(dout, p, mask):
    return np.where(mask, f64(dout) / (1 - p), 0.0)
