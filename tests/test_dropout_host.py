"""The dropout oracle's pins, and the host side of include/pair_dropout.h: symbols, layouts and refusals (no GPU)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import dropout as D
from paper_2603_14806_amd import trimul as T

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pair_dropout.h")


def test_philox_known_answers():
    """The published test vectors of Philox-4x32-10: zeros, ones, and the digits of pi."""
    vectors = [((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]
    for counter, key, want in vectors:
        assert tuple(int(w) for w in oracle.philox(np.array(counter, dtype=np.uint64), key)) == want


@pytest.mark.parametrize("share", ["none", "rows", "columns"])
def test_mask_of_a_tile_is_the_tile_of_the_mask(share):
    whole = oracle.keep(12, 20, 6, 0.3, 77, 5, share)
    tile = oracle.keep(5, 7, 6, 0.3, 77, 5, share, row0=4, col0=9, n_cols=20)
    assert np.array_equal(tile, whole[4:9, 9:16])
    if share == "rows":
        assert (whole == whole[:1]).all()
    if share == "columns":
        assert (whole == whole[:, :1]).all()
    assert not np.array_equal(whole, oracle.keep(12, 20, 6, 0.3, 78, 5, share))
    assert not np.array_equal(whole, oracle.keep(12, 20, 6, 0.3, 77, 6, share))


def test_rate_and_edges():
    m = oracle.keep(64, 64, 64, 0.25, 1, 0, "none")
    assert abs(m.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / m.size)          # five standard deviations
    assert oracle.keep(9, 9, 9, 0.0, 1, 0, "none").all()
    x, r = np.full((4, 4, 8), np.nan), np.ones((4, 4, 8))
    k = oracle.keep(4, 4, 8, 0.5, 3, 0, "none")
    out = oracle.dropout_add(x, r, 0.5, k)
    assert np.array_equal(np.isnan(out), k) and (out[~k] == 1).all()


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return D.lib()


def test_declared_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(pair_dropout_[a-z]+)\s*\(", text))
    assert names == set(D.SIGNATURES) and all(hasattr(lib, n) for n in names)
    assert ctypes.sizeof(D.PairDropoutView) == 8 * 8 + 3 * 4 + 4 + 8 + 2 * 8


def view(**kw):
    v = D.PairDropoutView(4, 6, 16, 0, 0, 6, 96, 96, T.TRI_MUL_F32, T.TRI_MUL_BF16, D.PAIR_DROPOUT_ROWS, 0.25, 1, 2)
    for k, x in kw.items():
        setattr(v, k, x)
    return ctypes.byref(v)


EINVAL, EUNSUPPORTED = T.TRI_MUL_EINVAL, T.TRI_MUL_EUNSUPPORTED


@pytest.mark.parametrize("change,code,word", [
    (dict(x_dtype=2), EINVAL, "dtype"), (dict(out_dtype=-1), EINVAL, "dtype"), (dict(share=3), EINVAL, "sharing"),
    (dict(share=-1), EINVAL, "sharing"), (dict(p=1.0), EINVAL, "p ="), (dict(p=-0.1), EINVAL, "p ="), (dict(p=float("nan")), EINVAL, "p ="),
    (dict(rows=-1), EINVAL, "negative"), (dict(cols=-1), EINVAL, "negative"), (dict(channels=-1), EINVAL, "negative"),
    (dict(row0=-1), EINVAL, "negative"), (dict(col0=-1), EINVAL, "negative"), (dict(col0=1), EINVAL, "outside"),
    (dict(n_cols=5), EINVAL, "outside"), (dict(ld_x=95), EINVAL, "row stride"), (dict(ld_out=95), EINVAL, "row stride"),
    (dict(ld_x=1 << 41), EINVAL, "2^40"), (dict(rows=1 << 41), EINVAL, "2^40"),
    (dict(cols=1 << 28, n_cols=1 << 28, ld_x=1 << 32, ld_out=1 << 32), EUNSUPPORTED, "2^31"),
    (dict(n_cols=1 << 60), EUNSUPPORTED, "2^62"), (dict(row0=1 << 58), EUNSUPPORTED, "2^62")])
def test_views_refused(lib, change, code, word):
    assert lib.pair_dropout_add(view(**change), 16, 16, 16, None) == code and word in T.last_error()
    assert lib.pair_dropout_backward(view(**change), 16, 16, None) == code and word in T.last_error()


def test_pointers_refused_and_empty_calls(lib):
    assert lib.pair_dropout_add(None, 16, 16, 16, None) == EINVAL
    for bad in ((None, 16, 16), (16, 16, None), (18, 16, 16), (16, 17, 16), (16, 16, 17)):
        assert lib.pair_dropout_add(view(), *bad, None) == EINVAL
    for bad in ((None, 16), (16, None), (17, 16), (16, 18)):
        assert lib.pair_dropout_backward(view(), *bad, None) == EINVAL
    for empty in (dict(rows=0), dict(cols=0), dict(channels=0)):
        assert lib.pair_dropout_add(view(**empty), None, None, None, None) == T.TRI_MUL_OK
        assert lib.pair_dropout_backward(view(**empty), None, None, None) == T.TRI_MUL_OK


def test_python_refusals():
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="GPU"):
        D.dropout_add(x)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        D.dropout_add(x.double())
    with pytest.raises(ValueError, match="rows"):
        D.dropout_backward(x[0])
