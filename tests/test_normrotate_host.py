"""The oracle's pins of the norms with rotation, and the host side of include/norm_rotate.h (no GPU)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import normrotate as O
from paper_2603_14806_amd import normrotate as N
from paper_2603_14806_amd import trimul as T

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "norm_rotate.h")


def test_by_hand():
    """Two pairs of (3, 4, 0, 0): rms 2.5, a quarter turn of the first pair and none of the second."""
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    phase = np.array([[1j, 1]])
    assert np.allclose(O.norm_rotate(x, phase, pairs="adjacent", eps=0.0), [-1.6, 1.2, 0, 0])
    assert np.allclose(O.norm_rotate(x, phase, pairs="halves", eps=0.0), [0, 1.6, 1.2, 0])
    # layer: centred (1.25, 2.25, -1.75, -1.75), variance 12.75 / 4; gain 2 on the first, shift 5 on the last
    assert np.allclose(O.norm_rotate(x + 7, phase, gain=[2, 1, 1, 1], shift=[0, 0, 0, 5.0], norm="layer", pairs="adjacent", eps=0.0),
                       np.array([-2.25, 2.5, -1.75, -1.75]) / np.sqrt(12.75 / 4) + [0, 0, 0, 5])
    assert np.allclose(O.phases([3], [0.5]), np.cos(1.5) + 1j * np.sin(1.5))


def test_relative_position_is_what_a_product_sees():
    """Products of turned rows depend on the distance of their positions alone."""
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 24))
    f = 10000.0 ** (-np.arange(8) / 8)
    for pairs in ("halves", "adjacent"):
        a = [(O.norm_rotate(q, O.phases([p], f), pairs=pairs) * O.norm_rotate(k, O.phases([p + 5], f), pairs=pairs)).sum() for p in (0, 17, 1000)]
        assert np.allclose(a, a[0], atol=1e-10)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
def test_gradients_against_differences(norm, pairs):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 2, 3, 2, 8))
    gain, shift = rng.standard_normal((2, 8))
    phase = O.phases(np.arange(6).reshape(2, 3), [1.0, 0.1])
    loss = lambda x, gain, shift: (O.norm_rotate(x, phase, gain, shift, norm, pairs) * dy).sum()
    dx, dgain, dshift = O.norm_rotate_backward(x, dy, phase, gain, norm, pairs)
    h = 1e-6
    for grad, at, name in ((dx, x, 0), (dgain, gain, 1), (dshift, shift, 2)):
        for i in [tuple(rng.integers(n) for n in grad.shape) for _ in range(12)]:
            args = [x, gain, shift]
            up, down = at.copy(), at.copy()
            up[i] += h
            down[i] -= h
            args[name] = up
            a = loss(*args)
            args[name] = down
            assert abs((a - loss(*args)) / (2 * h) - grad[i]) < 1e-7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return N.lib()


def test_declared_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\bint (norm_rotate_[a-z_]+)\s*\(", text))
    assert names == set(N.SIGNATURES) and all(hasattr(lib, n) for n in names)
    assert ctypes.sizeof(N.NormRotateView) == 2 * 8 + 7 * 4 + 4 + 3 * 8
    assert ctypes.sizeof(N.NormRotateSide) == 8 + 4 * 8 + 4 * 8 and ctypes.sizeof(N.NormRotateGrad) == 2 * 4 * 8 + 2 * 8


EINVAL, EUNSUPPORTED, ENOMEM = T.TRI_MUL_EINVAL, T.TRI_MUL_EUNSUPPORTED, T.TRI_MUL_ENOMEM


def changed(s, kw):
    for k, x in kw.items():
        setattr(s, k, x)
    return s


def view(**kw):
    return changed(N.NormRotateView(2, 10, 32, 16, T.TRI_MUL_BF16, T.TRI_MUL_F32, 0, 0, 1e-6, 16, 10, 16), kw)


def tensor(**kw):
    return changed(N.CrossAttnTensor(16, 10 * 4 * 32, 4 * 32, 32), kw)


def side(**kw):
    return changed(N.NormRotateSide(4, tensor(), 16, 16), kw)


def grad(**kw):
    return changed(N.NormRotateGrad(tensor(), tensor(), 16, 16), kw)


def calls(lib, v, q, k=None, yq=True, gq=True, x=True):
    """Return codes of the forward, the workspace's size and the backward."""
    n = ctypes.c_size_t()
    yq = tensor() if yq is True else yq
    gq = grad() if gq is True else gq
    yield lib.norm_rotate_forward(v, q, k, yq, tensor(), None)
    yield lib.norm_rotate_backward(v, q, k, gq, grad(), 256, 1 << 30, None)
    if x:
        yield lib.norm_rotate_backward_workspace_size(v, q, k, n)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(weight_dtype=-1), EINVAL, "dtype"), (dict(batch=-1), EINVAL, "negative"), (dict(n=-1), EINVAL, "negative"),
    (dict(batch=1 << 31), EUNSUPPORTED, "2^31"), (dict(n=1 << 31), EUNSUPPORTED, "2^31"), (dict(d=0, rot=0), EINVAL, "d ="), (dict(d=36), EINVAL, "d ="),
    (dict(d=264), EINVAL, "d ="), (dict(d=-8), EINVAL, "d ="), (dict(rot=-8), EINVAL, "rot"), (dict(rot=12), EINVAL, "rot"), (dict(rot=40), EINVAL, "rot"),
    (dict(layer=2), EINVAL, "layer"), (dict(adjacent=-1), EINVAL, "adjacent"), (dict(eps=0.0), EINVAL, "eps"), (dict(eps=-1.0), EINVAL, "eps"),
    (dict(eps=float("nan")), EINVAL, "eps"), (dict(eps=float("inf")), EINVAL, "eps"), (dict(freqs=None), EINVAL, "freqs"), (dict(freqs=20), EINVAL, "freqs"),
    (dict(positions=None), EINVAL, "positions"), (dict(positions=18), EINVAL, "positions"), (dict(positions_batch=-1), EINVAL, "positions")])
def test_views_refused(lib, change, code, word):
    for rc in calls(lib, view(**change), side()):
        assert rc == code and word in T.last_error()


def test_sides_refused(lib):
    for rc in calls(lib, None, side()):
        assert rc == EINVAL
    for rc in calls(lib, view(), None):
        assert rc == EINVAL and "neither" in T.last_error()
    for bad in (dict(heads=0), dict(heads=1025), dict(gain=24), dict(shift=8), dict(codes=16), dict(powers=16), dict(codes=24, powers=16)):
        for rc in calls(lib, view(), side(**bad)):
            assert rc == EINVAL
        for rc in calls(lib, view(), side(), side(**bad)):
            assert rc == EINVAL
    for bad, code in ((dict(data=24), EINVAL), (dict(token=132), EINVAL), (dict(head=24), EINVAL), (dict(batch=-1280), EINVAL), (dict(token=1 << 41), EUNSUPPORTED)):
        for rc in calls(lib, view(), side(x=tensor(**bad)), x=False):
            assert rc == code
        for rc in calls(lib, view(), side(), yq=tensor(**bad), gq=grad(dy=tensor(**bad)), x=False):
            assert rc == code
        assert lib.norm_rotate_backward(view(), side(), None, grad(dx=tensor(**bad)), None, 256, 1 << 30, None) == code
    for none in (dict(batch=0), dict(token=0), dict(head=0)):       # an input may be repeated, a result not
        assert lib.norm_rotate_forward(view(), side(), None, tensor(**none), None, None) == EINVAL
        assert lib.norm_rotate_backward(view(), side(), None, grad(dx=tensor(**none)), None, 256, 1 << 30, None) == EINVAL
    null = tensor(data=None)
    assert lib.norm_rotate_forward(view(), side(x=null), None, tensor(), None, None) == EINVAL
    assert lib.norm_rotate_forward(view(), side(), None, null, None, None) == EINVAL
    assert lib.norm_rotate_forward(view(), side(), None, None, None, None) == EINVAL
    for g in (None, grad(dy=null), grad(dx=null), grad(dgain=18), grad(dshift=17)):
        assert lib.norm_rotate_backward(view(), side(), None, g, None, 256, 1 << 30, None) == EINVAL
    assert lib.norm_rotate_backward(view(), side(x=null), None, grad(), None, 256, 1 << 30, None) == EINVAL
    held = dict(x=null, codes=16, powers=16)
    assert lib.norm_rotate_backward(view(), side(**held), side(), grad(), grad(), 256, 1 << 30, None) == EINVAL and "both" in T.last_error()
    assert lib.norm_rotate_backward(view(), side(), side(**held), grad(), grad(), 256, 1 << 30, None) == EINVAL and "both" in T.last_error()


def test_workspaces(lib):
    n = ctypes.c_size_t()
    assert lib.norm_rotate_backward_workspace_size(view(batch=50, n=1000), side(), side(), n) == 0 and 0 < n.value <= 16 << 20
    big = view(batch=50, n=1000)
    assert lib.norm_rotate_backward(big, side(), side(), grad(), grad(), 256, n.value - 1, None) == ENOMEM
    assert lib.norm_rotate_backward(big, side(), side(), grad(), grad(), 257, n.value, None) == EINVAL
    assert lib.norm_rotate_backward(big, side(), side(), grad(), grad(), None, n.value, None) == EINVAL
    assert lib.norm_rotate_backward_workspace_size(view(), side(), None, None) == EINVAL
    for empty in (dict(batch=0), dict(n=0)):
        v = view(positions=None, **empty)
        assert lib.norm_rotate_forward(v, side(x=tensor(data=None)), None, tensor(data=None), None, None) == T.TRI_MUL_OK


def test_python_refusals():
    x = torch.zeros(1, 2, 2, 8)
    f = N.frequencies(8, device="cpu")
    assert f.tolist() == [1.0, 0.1, 0.01, 10000.0 ** -0.75]
    with pytest.raises(ValueError, match="GPU"):
        N.norm_rotate(x, None)
    with pytest.raises(ValueError, match="neither"):
        N.norm_rotate(None, None)
    with pytest.raises(ValueError, match="rms"):
        N.norm_rotate(x, None, norm="l2")
    with pytest.raises(ValueError, match="halves"):
        N.norm_rotate(x, None, pairs="neighbours")
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        N.norm_rotate(x.half(), None)
    with pytest.raises(ValueError, match="heads"):
        N.norm_rotate_backward(x[0], None, x[0], None)


def test_more_values_than_counted_refused(lib):
    """Products of the sizes that wrap to zero in 64 bits are refused before anything is divided by them."""
    for batch, n in ((1 << 30, 1 << 30), (1 << 18, 1 << 18)):
        for rc in calls(lib, view(batch=batch, n=n, d=256, rot=0), side(heads=1024)):
            assert rc == EUNSUPPORTED and "2^44" in T.last_error()
