"""Host-side checks of include/cross_attn.h: exported symbols, struct layouts, and every refusal, none of which
touches a GPU (the pointers are never followed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2603_14806_amd import attention as A
from paper_2603_14806_amd import trimul as T

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "cross_attn.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return A.lib()


def test_declared_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(cross_attn_[a-z_]+)\s*\(", text))
    assert names == set(A.SIGNATURES)
    assert all(hasattr(lib, n) for n in names)
    assert ctypes.sizeof(A.CrossAttnTensor) == 4 * 8 and ctypes.sizeof(A.CrossAttnBias) == 4 * 8
    assert ctypes.sizeof(A.CrossAttnView) == 3 * 8 + 4 * 4 + 8 + 4 * 8 + 2 * 8     # scale is padded to 8


def view(**kw):
    w = A.CrossAttnView(2, 40, 50, 4, 2, 32, T.TRI_MUL_BF16, 0.5)
    for k, x in kw.items():
        setattr(w, k, x)
    return w


def tens(heads, tokens=50, **kw):
    t = A.CrossAttnTensor(1 << 12, tokens * heads * 32, heads * 32, 32)
    for k, x in kw.items():
        setattr(t, k, x)
    return t


def forward(lib, w, q=None, k=None, v=None, out=None, stats=None, ws=None, n=0):
    r = [ctypes.byref(x) if x is not None else None for x in (w, q or tens(4), k or tens(2), v or tens(2), out or tens(4))]
    return lib.cross_attn_forward(*r, stats, ws, n, None)


def backward(lib, w, stats=1 << 12, ws=1 << 12, n=1 << 20, dbias=None, **kw):
    names = ("q", "k", "v", "out"), ("dout", "dq", "dk", "dv")
    t = {x: tens(2 if x in ("k", "v", "dk", "dv") else 4) for x in names[0] + names[1]}
    t.update(kw)
    first, second = ([ctypes.byref(t[x]) if t[x] is not None else None for x in part] for part in names)
    return lib.cross_attn_backward(ctypes.byref(w), *first, stats, *second, None if dbias is None else ctypes.byref(dbias), ws, n, None)


EINVAL, EUNSUPPORTED, ENOMEM = T.TRI_MUL_EINVAL, T.TRI_MUL_EUNSUPPORTED, T.TRI_MUL_ENOMEM


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(batch=-1), EINVAL, "negative"), (dict(nq=-1), EINVAL, "negative"),
    (dict(nk=-3), EINVAL, "negative"), (dict(kv_heads=3), EINVAL, "multiple of kv_heads"), (dict(heads=0), EINVAL, "heads"),
    (dict(heads=2048), EUNSUPPORTED, "1024"), (dict(d=0), EUNSUPPORTED, "[8, 128]"), (dict(d=36), EUNSUPPORTED, "multiple of 8"),
    (dict(d=136), EUNSUPPORTED, "[8, 128]"), (dict(scale=0.0), EINVAL, "scale"), (dict(scale=-1.0), EINVAL, "scale"),
    (dict(scale=float("nan")), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"),
    (dict(nk=(1 << 24) + 1), EUNSUPPORTED, "2^24"), (dict(nq=(1 << 23) + 1), EUNSUPPORTED, "2^24"),
    (dict(batch=1 << 24), EUNSUPPORTED, "batch"), (dict(batch=1 << 23), EUNSUPPORTED, "too many"),
    (dict(mask=8, mask_batch=-1), EINVAL, "mask"),
    (dict(bias=A.CrossAttnBias(8, 0, 0, 56)), EINVAL, "aligned"), (dict(bias=A.CrossAttnBias(16, 0, 0, 48)), EINVAL, ">= nk"),
    (dict(bias=A.CrossAttnBias(16, 0, 0, 50)), EINVAL, "multiple of 8"), (dict(bias=A.CrossAttnBias(16, 0, 0, 1 << 25)), EINVAL, "2^24"),
    (dict(bias=A.CrossAttnBias(16, 4, 0, 56)), EINVAL, "strides"), (dict(bias=A.CrossAttnBias(16, 0, -8, 56)), EINVAL, "strides")])
def test_views_refused(lib, change, code, word):
    for call in (forward, backward):
        assert call(lib, view(**change)) == code
        assert word in T.last_error()
    n = ctypes.c_size_t()
    if word != "too many":
        assert lib.cross_attn_workspace_size(ctypes.byref(view(**change)), ctypes.byref(n)) == code
        assert lib.cross_attn_backward_workspace_size(ctypes.byref(view(**change)), ctypes.byref(n)) == code


@pytest.mark.parametrize("change,code,word", [
    (dict(data=None), EINVAL, "null"), (dict(data=(1 << 12) + 8), EINVAL, "aligned"), (dict(token=132), EINVAL, "16 bytes"),
    (dict(batch=-64), EINVAL, "16 bytes"), (dict(head=4), EINVAL, "16 bytes"), (dict(token=24), EINVAL, "below d"),
    (dict(token=1 << 23), EUNSUPPORTED, "2^23"), (dict(head=16), EINVAL, "below d"), (dict(batch=16), EINVAL, "below d")])
@pytest.mark.parametrize("name", ["q", "k", "v", "out", "dout", "dq", "dk", "dv"])
def test_tensors_refused(lib, name, change, code, word):
    t = tens(2 if name in ("k", "v", "dk", "dv") else 4, **change)
    if name in ("q", "k", "v", "out"):
        assert forward(lib, view(), **{name: t}) == code
        assert word in T.last_error()
    assert backward(lib, view(), **{name: t}) == code
    assert word in T.last_error() and name in T.last_error()


def test_null_and_workspace_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.cross_attn_workspace_size(None, ctypes.byref(n)) == EINVAL
    assert lib.cross_attn_workspace_size(ctypes.byref(view()), None) == EINVAL
    assert lib.cross_attn_backward_workspace_size(ctypes.byref(view()), None) == EINVAL
    assert lib.cross_attn_forward(None, None, None, None, None, None, None, 0, None) == EINVAL
    assert lib.cross_attn_forward(ctypes.byref(view()), None, None, None, None, None, None, 0, None) == EINVAL
    assert forward(lib, view(), out=tens(4, head=0)) == EINVAL            # outputs are not repeated
    few = view(batch=1, nq=1, nk=4000)
    assert lib.cross_attn_workspace_size(ctypes.byref(few), ctypes.byref(n)) == T.TRI_MUL_OK and n.value > 0
    assert forward(lib, few) == EINVAL and "workspace" in T.last_error()
    assert forward(lib, few, ws=1 << 12, n=n.value - 1) == ENOMEM
    assert forward(lib, few, ws=(1 << 12) + 16, n=n.value) == EINVAL
    assert lib.cross_attn_workspace_size(ctypes.byref(view(batch=300)), ctypes.byref(n)) == T.TRI_MUL_OK and n.value == 0
    assert backward(lib, view(), stats=None) == EINVAL and "stats" in T.last_error()
    assert backward(lib, view(), stats=(1 << 12) + 4) == EINVAL and "stats" in T.last_error()
    assert forward(lib, view(), stats=(1 << 12) + 8) == EINVAL and "stats" in T.last_error()
    assert lib.cross_attn_stats_size(ctypes.byref(view()), None) == EINVAL
    assert lib.cross_attn_stats_size(ctypes.byref(view()), ctypes.byref(n)) == T.TRI_MUL_OK
    assert n.value == 2 * 4 * 40 * 8 + 2 * 4 * 40 * 32 * 2     # 2560 bytes of sums are a multiple of 256
    assert lib.cross_attn_stats_size(ctypes.byref(view(dtype=T.TRI_MUL_F32, nq=41)), ctypes.byref(n)) == T.TRI_MUL_OK
    assert n.value == -(-2 * 4 * 41 * 8 // 256) * 256
    assert backward(lib, view(), ws=None) == EINVAL
    assert backward(lib, view(), n=16) == ENOMEM
    assert backward(lib, view(), dk=None) == EINVAL and "dk and dv" in T.last_error()
    assert backward(lib, view(), dq=tens(4, batch=0)) == EINVAL
    assert backward(lib, view(), dbias=A.CrossAttnBias(16, 0, 0, 56)) == EINVAL and "without a bias" in T.last_error()
    own = view(bias=A.CrossAttnBias(16, 4 * 40 * 56, 40 * 56, 56))
    for d in (A.CrossAttnBias(8, 0, 0, 56), A.CrossAttnBias(16, 4 * 40 * 56, 40 * 56, 52), A.CrossAttnBias(16, 0, 40 * 56, 56),
              A.CrossAttnBias(16, 4 * 40 * 56, 0, 56), A.CrossAttnBias(None, 4 * 40 * 56, 40 * 56, 56)):
        assert backward(lib, own, dbias=d) == EINVAL and "dbias" in T.last_error()


def test_empty_calls_are_done_at_once(lib):
    """Nothing to write, nothing launched: no batch entry or no query (and no key gradient to clear)."""
    empty = A.CrossAttnTensor(None, 0, 0, 0)
    assert forward(lib, view(batch=0), empty, empty, empty, empty) == T.TRI_MUL_OK
    assert forward(lib, view(nq=0), q=empty, out=empty) == T.TRI_MUL_OK
    t = dict.fromkeys(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), empty)
    assert backward(lib, view(batch=0), stats=None, **t) == T.TRI_MUL_OK


def test_python_refusals():
    """The torch side's checks come before the library is called, on CPU tensors as well."""
    q, k = torch.zeros(1, 4, 2, 32), torch.zeros(1, 6, 2, 32)
    with pytest.raises(ValueError, match="GPU"):
        A.cross_attention(q, k, k)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        A.cross_attention(q.half(), k.half(), k.half())
    with pytest.raises(ValueError, match=r"\[batch\]"):
        A.cross_attention(q[0], k, k)
