"""TriMul.residual on two streams at once, and captured at one size and replayed behind eager calls at another: the
results of calls made alone, bit for bit (the library's sums have one order)."""
import pytest
import torch

from paper_2603_14806_amd import synth
from tests.gpu_util import make_layer, needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


def test_two_streams_at_once():
    layer, _ = make_layer("bf16")
    zs = [synth.pair_tensor(n, dtype="bf16", seed=i, device="cuda") for i, n in enumerate((300, 300, 420, 129))]
    want = [layer.residual(z, None, "outgoing", 0.25, 7, i) for i, z in enumerate(zs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for turn in range(3):
        for i, z in enumerate(zs):
            s = streams[(i + turn) % 2]
            got.append((i, layer.residual(z, None, "outgoing", 0.25, 7, i, stream=s if turn else s.cuda_stream)))
    torch.cuda.synchronize()
    say(f"  {len(got)} residual calls on two streams")
    for i, y in got:
        assert torch.equal(y, want[i]), i
    layer.close()


def test_gradients_on_two_streams_at_once():
    layer, _ = make_layer("bf16")
    zs = [synth.pair_tensor(n, dtype="bf16", seed=i, device="cuda") for i, n in enumerate((200, 257))]
    douts = [synth.pair_tensor(z.shape[0], dtype="bf16", seed=20 + i, device="cuda") for i, z in enumerate(zs)]
    want = [layer.residual_backward(z, g, None, "incoming", 0.25, 7, 1) for z, g in zip(zs, douts)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [(i, layer.residual_backward(zs[i], douts[i], None, "incoming", 0.25, 7, 1, stream=streams[(i + turn) % 2]))
           for turn in range(2) for i in range(2)]
    torch.cuda.synchronize()
    for i, (dz, grads) in got:
        assert torch.equal(dz, want[i][0]) and all(torch.equal(grads[n], want[i][1][n]) for n in grads), i
    layer.close()


def test_replay_behind_calls_at_another_size():
    layer, _ = make_layer("bf16")
    z = synth.pair_tensor(96, dtype="bf16", seed=1, device="cuda")
    large = synth.pair_tensor(500, dtype="bf16", seed=2, device="cuda")
    layer.residual(z, p=0.25, seed=3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.residual(z, p=0.25, seed=3)
    for i in range(4):
        z.copy_(synth.pair_tensor(96, dtype="bf16", seed=10 + i, device="cuda"))
        layer.residual(large, p=0.25, seed=3)
        held = [torch.full((1 << 20,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(64)]   # memory given back is taken
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((h == 0x7f).all()) for h in held), i
        assert torch.equal(y, layer.residual(z, p=0.25, seed=3)), i
        del held
    layer.close()
