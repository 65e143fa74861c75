"""The rows of an attention bias are read up to a multiple of 8 values: the torch side refuses one whose last row's
padding is not its own memory.  No GPU: the checks come before any launch."""
import pytest
import torch

from paper_2603_14806_amd import attention as A


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
