"""fp64 CPU oracle for activations held in 8 bits.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import or call
this module.  It shares no code with the HIP library.

A group holds a power of two, the smallest 2^k (-127 <= k <= 121) in whose
steps its largest magnitude rounds to at most 127, and a whole number of steps
for each value (halves to even; what k = 121 leaves above 127 is cut off).
"""
import numpy as np

from .trimul import f64


def checkpoint8(x, group):
    """(codes [..., n] int8, powers [..., ceil(n / group)] uint8 = k + 127); 255 and codes 0 where a group is not finite."""
    x = f64(x)
    n = x.shape[-1]
    codes = np.zeros(x.shape, dtype=np.int8)
    powers = np.zeros(x.shape[:-1] + (-(-n // group),), dtype=np.uint8)
    for g in range(powers.shape[-1]):
        part = x[..., g * group:(g + 1) * group]
        finite = np.isfinite(part).all(axis=-1)
        part = np.where(finite[..., None], part, 0.0)
        top = np.abs(part).max(axis=-1)
        k = np.full(top.shape, -127)
        while True:                                  # (from the smallest power upwards: no logarithm to be near a border of)
            over = (np.rint(top * 2.0 ** -k) > 127) & (k < 121)
            if not over.any():
                break
            k = np.where(over, k + 1, k)
        codes[..., g * group:(g + 1) * group] = np.clip(np.rint(part * 2.0 ** -k[..., None]), -127, 127)
        powers[..., g] = np.where(finite, k + 127, 255)
    return codes, powers


def checkpoint8_values(codes, powers, group):
    scale = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return codes.astype(np.float64) * np.repeat(scale, group, axis=-1)[..., :codes.shape[-1]]
