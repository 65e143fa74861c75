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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,nq", [(2, 9), (70, 140)])
def test_bias_of_minus_infinity_is_weight_zero(B, nq, dtype):
    """Keys that every query's bias removes, with values of 1e30 (finite, and so are their products with dout):
    the bits of the same keys absent by the mask, gradients included."""
    g = torch.Generator().manual_seed(2)
    q, dout = (torch.randn((B, nq, 4, 32), generator=g).to(dtype).cuda() for _ in range(2))
    k, v = (torch.randn((B, 80, 4, 32), generator=g).to(dtype).cuda() for _ in range(2))
    mask = (torch.rand((B, 80), generator=g) < 0.6).to(torch.uint8).cuda()
    gone = mask == 0
    v[gone] = 1e30
    bias = torch.randn((B, 4, nq, 80), generator=g).to(dtype).cuda()
    low = torch.where(gone[:, None, None, :], torch.full_like(bias, -float("inf")), bias)
    results = []
    for b, m in ((low, None), (bias, mask)):
        out, stats = A.cross_attention(q, k, v, b, m, return_stats=True)
        results.append((out,) + A.cross_attention_backward(q, k, v, out, stats, dout, b, m))
    for n, a, b in zip(("out", "dq", "dk", "dv", "dbias"), *results):
        assert torch.equal(a, b), n
