"""The rows of an attention bias are read up to a multiple of 8 values: the torch side refuses one whose last row's
padding is not its own memory.  No GPU: the checks come before any launch."""
import ctypes
import os

import pytest
import torch

from paper_2603_14806_amd import attention as A
from paper_2603_14806_amd import trimul as T


def check(t, batch, heads, nq, nk):
    return A._checked_bias(t, batch, heads, nq, nk)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_past_the_end_is_refused(dtype):
    per = 16 // torch.empty((), dtype=dtype).element_size()
    # rows 264 values apart, a view that starts at the second 16 bytes: in float32 the last row's 264 values end 4 past
    # the tensor's
    late = torch.zeros(1, 2, 9, 264, dtype=dtype)[..., per:]
    if dtype == torch.float32:
        with pytest.raises(ValueError, match="padded"):
            check(late, 1, 2, 9, 260)
        assert check(late[..., :252], 1, 2, 9, 252).row == 264
    else:
        assert check(late, 1, 2, 9, 256).row == 264
    # a last row cut off at its keys
    cut = torch.zeros(9 * 264 - 7, dtype=dtype).as_strided((1, 1, 9, 257), (9 * 264, 9 * 264, 264, 1))
    with pytest.raises(ValueError, match="padded"):
        check(cut, 1, 1, 9, 257)
    with pytest.raises(ValueError, match="padded"):
        check(cut[0], 1, 1, 9, 257)


def test_padded_views_are_taken():
    full = torch.zeros(2, 3, 5, 24)
    for t, batch, heads in ((full[..., :20], 2, 3), (full[..., 4:20], 2, 3), (full[:1, :1, :, :17], 7, 4), (full[0, ..., :20], 6, 3)):
        b = check(t, batch, heads, 5, t.shape[-1])
        assert b.data == t.data_ptr() and b.row == 24
    assert check(torch.zeros(1, 3, 0, 8), 2, 3, 0, 8).data is None
    for t in (full[..., :20], full[..., ::2]):
        with pytest.raises(ValueError):
            check(t, 2, 3, 5, 12)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        from paper_2603_14806_amd import build
        build.build()
    return A.lib()


@pytest.mark.parametrize("sizes,bias,ok", [
    (dict(nq=1), (0, 56, 50), True), (dict(nq=1), (0, 56, 3), True), (dict(nq=2), (0, 56, 50), False), (dict(nq=2), (0, 56, 3), False),
    (dict(batch=1), (5, 56, 56), True), (dict(batch=2), (5, 56, 56), False),
    (dict(heads=1, kv_heads=1), (8, 3, 56), True), (dict(nq=1), (0, 57, 50), False)])
def test_strides_of_axes_of_length_one_are_not_looked_at(lib, sizes, bias, ok):
    w = A.CrossAttnView(1, 9, 50, 4, 2, 32, T.TRI_MUL_BF16, 0.5, A.CrossAttnBias(1 << 12, *bias))
    for k, x in sizes.items():
        setattr(w, k, x)
    n = ctypes.c_size_t()
    for size in (lib.cross_attn_workspace_size, lib.cross_attn_backward_workspace_size):
        assert size(ctypes.byref(w), ctypes.byref(n)) == (T.TRI_MUL_OK if ok else T.TRI_MUL_EINVAL)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU visible")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk", [(1, 4, 2), (3, 2, 2), (1, 1, 1)])
def test_one_query_with_any_row_stride(B, H, Hk, dtype):
    """torch names the stride of an axis of length 1 as it likes: 257 for the rows below, 264 values apart in truth."""
    from tests.test_gpu_crossattn import call, check as against, cuda, make
    x = cuda(make(B, 1, 257, H, Hk, 32, dtype, (B, H), "random"))
    want, _ = call(x)
    rows = torch.zeros(B, H, 264, dtype=x["q"].dtype, device="cuda")
    rows[..., :257] = x["bias"][:, :, 0]
    y = dict(x, bias=rows[..., :257].unsqueeze(2))
    assert y["bias"].stride(2) == 257 and y["bias"].shape == x["bias"].shape
    got, _ = call(y)
    against(got, y, f"single query {dtype}", dtype)
    assert all(torch.equal(got[n], want[n]) for n in want)
    with pytest.raises(ValueError, match="padded"):            # 257 values and nothing behind them
        A.cross_attention(x["q"], x["k"], x["v"], torch.zeros(1, 1, 1, 257, dtype=x["q"].dtype, device="cuda"))
