"""Cross attention at the edges of what its documentation allows and refuses."""
import pytest
import torch

from paper_2603_14806_amd import attention as A
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("d", [0, 4, 12, 136])
def test_widths_refused(d):
    q, k = torch.zeros(1, 3, 2, d, device="cuda"), torch.zeros(1, 5, 2, d, device="cuda")
    with pytest.raises(T.TriMulError) as e:
        A.cross_attention(q, k, k)
    assert e.value.code == T.TRI_MUL_EUNSUPPORTED


def test_no_heads_refused():
    q, k = torch.zeros(1, 3, 0, 32, device="cuda"), torch.zeros(1, 5, 0, 32, device="cuda")
    with pytest.raises(T.TriMulError) as e:
        A.cross_attention(q, k, k)
    assert e.value.code == T.TRI_MUL_EINVAL
