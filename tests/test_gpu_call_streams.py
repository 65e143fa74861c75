"""Wrapper calls with a stream argument: their workspaces belong to that stream, so that what is allocated on the current
one right behind them does not share memory with kernels still running.  Equal to the calls made alone, bit for bit."""
import pytest
import torch

from paper_2603_14806_amd import synth
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import make_layer, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


def test_gradients_and_outer_product_mean_on_side_streams():
    layer, _ = make_layer("bf16")
    n = 200
    z = synth.pair_tensor(n, dtype="bf16", seed=1, device="cuda")
    dout = torch.randn((n, n, 128), generator=torch.Generator().manual_seed(2)).cuda()
    g = torch.Generator().manual_seed(3)
    op = T.OuterProductMean(torch.randn((128, 1024), generator=g) / 32)
    a, b = (torch.randn((40, n, 32), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    A, B = layer.project(z)
    dC = layer.contract(A, B, n)

    def calls(stream):
        dz, grads = layer.backward(z, dout, None, "outgoing", stream=stream)
        panels, results = layer.project(z, stream=stream), layer.contract_backward(dC, A, B, n, stream=stream)
        return [dz, *grads.values(), op.forward(a, b, None, stream=stream)], panels, (*results, layer.contract(A, B, n, stream=stream))

    def values(r):
        """Without the layouts' padding, which is unspecified."""
        return r[0] + [T.panel_to_dense(t, n) for t in r[1]] + [T.result_to_dense(t, n) for t in r[2]]
    want = values(calls(None))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        got, held = [], []
        for s in streams:
            got.append(calls(s if turn else s.cuda_stream))
            held += [torch.full((1 << 22,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for r in got:
            assert all(torch.equal(x, y) for x, y in zip(values(r), want)), turn
        assert all(bool((h == 0xff).all()) for h in held)
    op.close()
    layer.close()
