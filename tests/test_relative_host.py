"""Buckets, the oracle's pins of the relative position bias, and the host side of include/relative_bias.h (no GPU)."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import relative as O
from paper_2603_14806_amd import relative as R
from paper_2603_14806_amd import trimul as T

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "relative_bias.h")


def lut_of(b):
    return b.lut.tolist()


def test_clipped():
    b = R.Buckets.clipped(3, other=True, device="cpu")
    assert lut_of(b) == list(range(7)) and b.reach == 3 and b.rows == 8
    assert lut_of(R.Buckets.clipped(0, device="cpu")) == [0]
    assert R.Buckets.clipped(127, other=True, device="cpu").rows == 256


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("n,reach", [(32, 128), (8, 100), (64, 1000), (48, 4095), (12, 7)])
def test_logarithmic(n, reach, both):
    b = R.Buckets.logarithmic(n, reach, both=both, device="cpu")
    per = n // 2 if both else n
    single = per // 2
    lut = lut_of(b)
    assert len(lut) == 2 * reach + 1
    for r in range(reach + 1):
        want = O.log_bucket(r, single, per - single, reach)
        assert lut[reach - r] == want
        assert lut[reach + r] == (want if r == 0 else per + want if both else 0)
        # the logarithm itself, where it is not next to a border
        x = math.log(max(r, 1) / single) / math.log(reach / single) * (per - single)
        if r >= single and abs(x - round(x)) > 1e-9:
            assert want == min(per - 1, single + int(x))
    assert b.rows == max(lut) + 1 and (max(lut) == n - 1 or reach < 2 * n)


def test_worked_borders():
    """32 buckets up to 128: 8 single distances, then 8 * 2^(k / 2): 8, 12, 16, 23, 32, 46, 64, 91."""
    lut = lut_of(R.Buckets.logarithmic(32, 128, device="cpu"))
    first = [next(r for r in range(129) if lut[128 - r] == b) for b in range(16)]
    assert first == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


def test_refused_buckets():
    for bad in ([0, 1], [0] * 8193, [256], [-1], []):
        with pytest.raises(ValueError):
            R.Buckets(bad, device="cpu")
    with pytest.raises(ValueError):
        R.Buckets([255], other=True, device="cpu")
    for bad in ((2, 100, True), (31, 100, True), (32, 8, True), (1, 100, False), (32, 4096, True)):
        with pytest.raises(ValueError):
            R.Buckets.logarithmic(*bad, device="cpu")


def test_oracle_by_hand():
    lut, q, k = [5, 6, 7], [10, -2 ** 31], [9, 10, 12, 2 ** 31 - 1]
    b = O.buckets(lut, 9, q, k)
    assert b.tolist() == [[5, 6, 7, 7], [7, 7, 7, 7]]
    assert O.buckets(lut, 9, q, k, [1, 2], [1, 1, 2, 2]).tolist() == [[5, 6, 8, 8], [8, 8, 7, 7]]
    table = np.arange(18).reshape(9, 2)
    assert O.relative_bias(table, b)[1].tolist() == [[11, 13, 15, 15], [15] * 4]
    g = O.table_gradient(np.ones((2, 4, 2)), b, 9)
    assert g[:, 0].tolist() == [0, 0, 0, 0, 0, 1, 1, 6, 0]
    assert np.array_equal(O.relative_pair(table, b, np.ones((2, 4, 2)))[..., 0], O.relative_bias(table, b)[0] + 1)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return R.lib()


def test_declared_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\bint (relative_[a-z_]+)\s*\(", text))
    assert names == set(R.SIGNATURES) and all(hasattr(lib, n) for n in names)
    assert ctypes.sizeof(R.RelativeView) == 3 * 8 + 5 * 4 + 4 + 9 * 8


EINVAL, EUNSUPPORTED, ENOMEM = T.TRI_MUL_EINVAL, T.TRI_MUL_EUNSUPPORTED, T.TRI_MUL_ENOMEM


def view(**kw):
    v = R.RelativeView(2, 10, 20, 4, T.TRI_MUL_BF16, T.TRI_MUL_F32, 9, 4, 16, 16, 16, 10, 20)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


def bias(**kw):
    b = R.CrossAttnBias(16, 4 * 10 * 24, 10 * 24, 24)
    for k, x in kw.items():
        setattr(b, k, x)
    return b


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(table_dtype=-1), EINVAL, "dtype"), (dict(batch=-1), EINVAL, "negative"),
    (dict(nq=-1), EINVAL, "negative"), (dict(nk=-1), EINVAL, "negative"), (dict(heads=0), EINVAL, "1024"),
    (dict(heads=1025), EINVAL, "1024"), (dict(buckets=0), EINVAL, "buckets"), (dict(buckets=257), EINVAL, "buckets"),
    (dict(reach=-1), EINVAL, "reach"), (dict(reach=4096), EINVAL, "reach"), (dict(nq=1 << 24), EUNSUPPORTED, "2^24"),
    (dict(nk=1 << 24), EUNSUPPORTED, "2^24"), (dict(lut=None), EINVAL, "lut"), (dict(pos_q=None), EINVAL, "positions"),
    (dict(pos_k=None), EINVAL, "positions"), (dict(pos_k=18), EINVAL, "aligned"), (dict(seg_q=16), EINVAL, "segments"),
    (dict(seg_k=16), EINVAL, "segments")])
def test_views_refused(lib, change, code, word):
    n = ctypes.c_size_t()
    v, w = view(**change), view(**{"batch": 1, **change})
    assert lib.relative_bias(v, 16, None, bias(), None) == code and word in T.last_error()
    assert lib.relative_bias_backward_workspace_size(v, n) == code and word in T.last_error()
    assert lib.relative_bias_backward(v, bias(), 16, 256, 1 << 30, None) == code and word in T.last_error()
    assert lib.relative_pair(w, 16, None, 0, 16, 1 << 20, None) == code and word in T.last_error()
    assert lib.relative_pair_backward_workspace_size(w, n) == code and word in T.last_error()
    assert lib.relative_pair_backward(w, 16, 1 << 20, 16, 256, 1 << 30, None) == code and word in T.last_error()


def test_strides_and_pointers_refused(lib):
    assert lib.relative_bias(None, 16, None, bias(), None) == EINVAL
    assert lib.relative_bias(view(pos_q_batch=-1), 16, None, bias(), None) == EINVAL
    for table in (None, 18):
        assert lib.relative_bias(view(), table, None, bias(), None) == EINVAL
        assert lib.relative_pair(view(batch=1), table, None, 0, 16, 80, None) == EINVAL
    for out in (None, bias(data=None), bias(data=17), bias(row=19), bias(head=0), bias(batch=0), bias(row=-24)):
        assert lib.relative_bias(view(), 16, None, out, None) == EINVAL
    assert lib.relative_bias(view(), 16, None, bias(batch=1 << 41), None) == EUNSUPPORTED
    for base in (bias(data=None), bias(data=17), bias(row=-1)):
        assert lib.relative_bias(view(), 16, base, bias(), None) == EINVAL
    for args in ((None, 80), (17, 80), (16, 79)):
        assert lib.relative_pair(view(batch=1), 16, None, 0, *args, None) == EINVAL
        assert lib.relative_pair_backward(view(batch=1), *args, 16, 256, 1 << 30, None) == EINVAL
    assert lib.relative_pair(view(), 16, None, 0, 16, 80, None) == EINVAL and "batch" in T.last_error()
    assert lib.relative_pair(view(batch=1), 16, 16, 79, 16, 80, None) == EINVAL
    n = ctypes.c_size_t()
    assert lib.relative_bias_backward_workspace_size(view(), n) == 0 and n.value >= 4 * 2 * 4 * 9
    assert lib.relative_bias_backward(view(), bias(), 16, 256, n.value - 1, None) == ENOMEM
    assert lib.relative_bias_backward(view(), bias(), 16, 257, n.value, None) == EINVAL
    assert lib.relative_bias_backward(view(), bias(), 16, None, n.value, None) == EINVAL
    for dtable in (None, 18):
        assert lib.relative_bias_backward(view(), bias(), dtable, 256, n.value, None) == EINVAL
        assert lib.relative_pair_backward(view(batch=1), 16, 80, dtable, 256, 1 << 30, None) == EINVAL
    assert lib.relative_pair_backward_workspace_size(view(batch=1), n) == 0 and n.value > 0
    assert lib.relative_pair_backward(view(batch=1), 16, 80, 16, 256, n.value - 1, None) == ENOMEM


def test_empty_forwards(lib):
    for empty in (dict(nq=0), dict(nk=0), dict(batch=0)):
        assert lib.relative_bias(view(**empty), None, None, None, None) == T.TRI_MUL_OK
    for empty in (dict(nq=0), dict(nk=0)):
        assert lib.relative_pair(view(batch=1, **empty), None, None, 0, None, 0, None) == T.TRI_MUL_OK


def test_workspaces_stay_small(lib):
    """Partial sums of a tile grid, not of the pairs: below 64 MB for 66 buckets of 128 channels, whatever the shape."""
    n = ctypes.c_size_t()
    for nq, nk in ((1, 1), (1, 1 << 23), (1 << 23, 1), (3, 1 << 20), (1000, 1000), (16384, 16384), (100000, 17)):
        assert lib.relative_pair_backward_workspace_size(view(batch=1, nq=nq, nk=nk, heads=128, buckets=66, reach=32), n) == 0
        assert n.value < 64 << 20, (nq, nk, n.value)
        assert lib.relative_bias_backward_workspace_size(view(batch=1, nq=nq, nk=nk, heads=16, buckets=66, reach=32), n) == 0
        assert n.value < 8 << 20


def test_python_refusals():
    p, b = torch.zeros(4, dtype=torch.int32), R.Buckets.clipped(1, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        R.relative_bias(torch.zeros(3, 2), b, p, p)
    with pytest.raises(ValueError, match="Buckets"):
        R.relative_pair(torch.zeros(3, 2), [0, 1, 2], p, p)
    with pytest.raises(ValueError, match="heads"):
        R.relative_bias(torch.zeros(3), b, p, p)
    with pytest.raises(ValueError, match="batch"):
        R.relative_bias_backward(torch.zeros(4, 4), b, p, p)
    with pytest.raises(ValueError, match="channels"):
        R.relative_pair_backward(torch.zeros(4, 4), b, p, p)


def test_more_values_than_counted_refused(lib):
    """Products of the sizes that wrap to zero in 64 bits are refused before anything is divided by them."""
    n = ctypes.c_size_t()
    for size in (1 << 23, 1 << 13):
        v = view(batch=size, nq=size, nk=size, heads=1024)
        far = bias(batch=1 << 30, head=1 << 30, row=1 << 30)
        assert lib.relative_bias(v, 16, None, far, None) == EUNSUPPORTED and "2^48" in T.last_error()
        assert lib.relative_bias_backward_workspace_size(v, n) == EUNSUPPORTED and "2^48" in T.last_error()
        assert lib.relative_bias_backward(v, far, 16, 256, 1 << 30, None) == EUNSUPPORTED and "2^48" in T.last_error()
    v = view(batch=1, nq=1 << 23, nk=1 << 23, heads=1024)
    assert lib.relative_pair(v, 16, None, 0, 16, 1 << 33, None) == EUNSUPPORTED and "2^48" in T.last_error()
    assert lib.relative_pair_backward(v, 16, 1 << 33, 16, 256, 1 << 30, None) == EUNSUPPORTED and "2^48" in T.last_error()
