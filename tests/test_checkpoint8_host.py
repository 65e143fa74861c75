"""The oracle's pins of activations in 8 bits, and the host side of include/checkpoint8.h (no GPU)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import checkpoint8 as C
from paper_2603_14806_amd import trimul as T

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "checkpoint8.h")


def test_worked_values():
    """m = 1.99: 127.36 rounds to 127; m = 1.9921875: the tie 127.5 rounds to 128, one power more; zeros; not finite."""
    x = np.array([[1.99, -1.0, 0.5 / 64, 1.5 / 64], [1.9921875, -1.0, 0.5, 3 / 64], [0, 0, 0, -0.0], [1, np.inf, 2, 3], [1, np.nan, 2, 3]])
    codes, powers = oracle.checkpoint8(x, 8)
    assert powers[:, 0].tolist() == [127 - 6, 127 - 5, 0, 255, 255]
    assert codes.tolist() == [[127, -64, 0, 2], [64, -32, 16, 2], [0] * 4, [0] * 4, [0] * 4]
    v = oracle.checkpoint8_values(codes, powers, 8)
    assert v[0].tolist() == [127 / 64, -1, 0, 2 / 64] and np.isnan(v[3:]).all() and (v[2] == 0).all()


def test_error_and_idempotence():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 100)) * np.exp(rng.standard_normal(100))
    for group in (8, 24, 32, 128):
        codes, powers = oracle.checkpoint8(x, group)
        v = oracle.checkpoint8_values(codes, powers, group)
        top = np.repeat(np.maximum.reduceat(np.abs(x), range(0, 100, group), axis=1), group, axis=1)[:, :100]
        assert (np.abs(v - x) <= top / 127).all() and np.abs(codes.astype(int)).max() <= 127
        again = oracle.checkpoint8(v, group)
        assert np.array_equal(oracle.checkpoint8_values(*again, group), v)
        wide = torch.from_numpy(v).to(torch.bfloat16).double().numpy()
        assert np.array_equal(wide, v)                                                        # exact in bf16
    tiny = np.full((1, 8), 2.0 ** -140)
    assert oracle.checkpoint8(tiny, 8)[1][0, 0] == 0


def test_error_at_the_ends_of_the_range():
    """Where k is held at -127 (amax below 127 2^-128) half a step is 2^-128, which may be more than amax / 127, and from
    amax = 2^-128 down nothing is left; where it is held at 121, a step."""
    rng = np.random.default_rng(2)
    border = 127 * 2.0 ** -128
    top = np.concatenate([2.0 ** rng.uniform(-149, -118, 400), border * np.array([1 - 2.0 ** -20, 1, 1 + 2.0 ** -20]), 2.0 ** np.arange(-149.0, -120)])
    x = (top[:, None] * rng.uniform(-1, 1, (len(top), 8)))
    x[:, 3] = top
    x = x.astype(np.float32).astype(np.float64)
    top = np.abs(x).max(-1)
    codes, powers = oracle.checkpoint8(x, 8)
    error = np.abs(oracle.checkpoint8_values(codes, powers, 8) - x).max(-1)
    small = top < border
    assert (powers[small, 0] == 0).all() and (error[small] <= 2.0 ** -128).all() and (error[~small] <= top[~small] / 127).all()
    assert (error[small] > top[small] / 127).any() and (codes[top <= 2.0 ** -128] == 0).all()
    big = float(np.finfo(np.float32).max)
    x = rng.uniform(0.99, 1, (50, 8)) * big
    codes, powers = oracle.checkpoint8(x, 8)
    assert (powers == 248).all() and (np.abs(oracle.checkpoint8_values(codes, powers, 8) - x) <= 2.0 ** 121).all()


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return C.lib()


def test_declared_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(checkpoint8_[a-z]+)\s*\(", text))
    assert names == set(C.SIGNATURES) and all(hasattr(lib, n) for n in names)
    assert ctypes.sizeof(C.Checkpoint8View) == 3 * 8 + 2 * 4


EINVAL, EUNSUPPORTED = T.TRI_MUL_EINVAL, T.TRI_MUL_EUNSUPPORTED


def view(**kw):
    v = C.Checkpoint8View(4, 96, 96, T.TRI_MUL_BF16, 32)
    for k, x in kw.items():
        setattr(v, k, x)
    return ctypes.byref(v)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(group=0), EINVAL, "group"), (dict(group=12), EINVAL, "group"), (dict(group=264), EINVAL, "group"),
    (dict(group=-8), EINVAL, "group"), (dict(rows=-1), EINVAL, "negative"), (dict(n=-1), EINVAL, "negative"), (dict(ld=95), EINVAL, "stride"),
    (dict(ld=-96), EINVAL, "stride"), (dict(rows=1 << 40), EUNSUPPORTED, "2^40"), (dict(n=1 << 40, ld=1 << 40), EUNSUPPORTED, "2^40"),
    (dict(ld=1 << 40), EUNSUPPORTED, "2^40"), (dict(rows=1 << 39, ld=1 << 39), EUNSUPPORTED, "2^62"),
    (dict(rows=1 << 36), EUNSUPPORTED, "too many")])
def test_views_refused(lib, change, code, word):
    assert lib.checkpoint8_pack(view(**change), 16, 16, 16, None) == code and word in T.last_error()
    assert lib.checkpoint8_unpack(view(**change), 16, 16, 16, None) == code and word in T.last_error()


def test_pointers_refused_and_empty_calls(lib):
    assert lib.checkpoint8_pack(None, 16, 16, 16, None) == EINVAL
    for bad in ((None, 16, 16), (16, None, 16), (16, 16, None), (17, 16, 16)):
        assert lib.checkpoint8_pack(view(), *bad, None) == EINVAL
    for bad in ((None, 16, 16), (16, None, 16), (16, 16, None), (16, 16, 17)):
        assert lib.checkpoint8_unpack(view(), *bad, None) == EINVAL
    for empty in (dict(rows=0), dict(n=0)):
        assert lib.checkpoint8_pack(view(**empty), None, None, None, None) == T.TRI_MUL_OK
        assert lib.checkpoint8_unpack(view(**empty), None, None, None, None) == T.TRI_MUL_OK


def test_python_refusals():
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="GPU"):
        C.pack(x)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        C.pack(x.half())


def test_codes_that_do_not_fit_refused():
    """A Checkpoint8 of one's own (read from a file, cut from another): what the kernels assume of it is checked."""
    def codes(*shape, dtype=torch.int8):
        return torch.zeros(shape, dtype=dtype)

    def powers(*shape, dtype=torch.uint8):
        return torch.zeros(shape, dtype=dtype)
    ok = C.Checkpoint8(codes(3, 5, 40), powers(3, 5, 2), 32, torch.bfloat16)
    assert ok.shape == (3, 5, 40)
    C.Checkpoint8(codes(0, 40), powers(0, 2), 32, torch.float32)
    for c, p, group, dtype in ((codes(3, 40), powers(3, 1), 32, torch.float32), (codes(3, 40), powers(4, 2), 32, torch.float32),
                               (codes(3, 40, dtype=torch.uint8), powers(3, 2), 32, torch.float32), (codes(3, 40), powers(3, 2, dtype=torch.int8), 32, torch.float32),
                               (codes(3, 40), powers(3, 2), 32, torch.float16), (codes(3, 40), powers(3, 2), 0, torch.float32), (codes(3, 40), powers(3, 2), 36, torch.float32),
                               (codes(3, 40), powers(3, 2), 264, torch.float32), (codes(3, 80)[:, ::2], powers(3, 2), 32, torch.float32),
                               (codes(3, 40), powers(3, 4)[:, :2], 32, torch.float32)):
        with pytest.raises(ValueError):
            C.Checkpoint8(c, p, group, dtype)
