"""Offsets past 2^31 elements, and calls whose LDS is above 64 KB inside a captured graph: the norms with rotation, the
relative position bias and the 8-bit checkpoints on views of one large buffer give what they give on small tensors."""
import pytest
import torch

from paper_2603_14806_amd import checkpoint8 as C
from paper_2603_14806_amd import normrotate as N
from paper_2603_14806_amd import relative as R
from tests.gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

FAR = (1 << 31) + 64


@pytest.fixture(scope="module")
def buffer():
    flat = torch.empty(FAR + (1 << 16), dtype=torch.bfloat16, device="cuda")
    yield flat
    del flat
    torch.cuda.empty_cache()


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def far(buffer, x, strides, offset=0):
    v = buffer.as_strided(x.shape, strides, offset)
    v.copy_(x)
    return v


@pytest.mark.parametrize("axis", ["batch", "token", "head"])
def test_norm_rotate(buffer, axis):
    x, dy = normal((2, 2, 2, 32), 1), normal((2, 2, 2, 32), 2)
    strides = {"batch": (FAR, 1024, 64, 1), "token": (1024, FAR, 64, 1), "head": (1024, 64, FAR, 1)}[axis]
    pos, freqs = torch.arange(2, dtype=torch.int32).cuda(), N.frequencies(32)
    want = N.norm_rotate(x, None, pos, freqs)[0]
    back = N.norm_rotate_backward(x, None, dy, None, pos, freqs)[0]
    v = far(buffer, x, strides)
    assert torch.equal(N.norm_rotate(v, None, pos, freqs)[0], want)
    assert torch.equal(N.norm_rotate_backward(v, None, dy, None, pos, freqs)[0], back)
    w = far(buffer, dy, strides, 4096)
    assert torch.equal(N.norm_rotate_backward(x, None, w, None, pos, freqs)[0], back)
    N.norm_rotate(x, None, pos, freqs, out_q=w)
    assert torch.equal(w, want) and torch.equal(v, x)


@pytest.mark.parametrize("axis", ["batch", "head", "row"])
def test_relative_bias(buffer, axis):
    b = R.Buckets.clipped(4)
    base, table = normal((2, 2, 2, 40), 1), normal((b.rows, 2), 2)
    strides = {"batch": (FAR, 1024, 64, 1), "head": (1024, FAR, 64, 1), "row": (1024, 64, FAR, 1)}[axis]
    pq, pk = torch.arange(2, dtype=torch.int32).cuda() + 20, torch.arange(40, dtype=torch.int32).cuda()
    want, grad = R.relative_bias(table, b, pq, pk, base=base), R.relative_bias_backward(base, b, pq, pk)
    v = far(buffer, base, strides)
    assert torch.equal(R.relative_bias(table, b, pq, pk, base=v), want) and torch.equal(R.relative_bias_backward(v, b, pq, pk), grad)
    assert R.relative_bias(table, b, pq, pk, base=v, out=v) is v and torch.equal(v, want)


def test_relative_pair_and_checkpoint(buffer):
    b = R.Buckets.clipped(4)
    base, table = normal((2, 40, 64), 1), normal((b.rows, 64), 2)
    pq, pk = torch.arange(2, dtype=torch.int32).cuda() + 20, torch.arange(40, dtype=torch.int32).cuda()
    want, grad = R.relative_pair(table, b, pq, pk, base=base), R.relative_pair_backward(base, b, pq, pk)
    v = far(buffer, base, (FAR, 64, 1))
    assert torch.equal(R.relative_pair(table, b, pq, pk, base=v), want) and torch.equal(R.relative_pair_backward(v, b, pq, pk), grad)
    flat = buffer.as_strided((2, 40 * 64), (FAR, 1), 0)
    c = C.pack(flat)
    assert torch.equal(c.codes, C.pack(base.reshape(2, -1)).codes)
    flat.fill_(7.0)
    assert c.unpack(out=flat) is flat and torch.equal(flat, C.pack(base.reshape(2, -1)).unpack())


def test_codes_past_two_gigabytes():
    """2^31 + values in one call of the checkpoint: its last groups."""
    n = (1 << 31) + 4096
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[-5000:] = normal((5000,), 3)
    c = C.pack(x, 64)
    part = C.pack(x[-4096:], 64)
    assert torch.equal(c.codes[-4096:], part.codes) and torch.equal(c.powers[-64:], part.powers) and int(c.codes[:1 << 20].abs().max()) == 0
    assert torch.equal(c.unpack()[-4096:], part.unpack())
    del x, c
    torch.cuda.empty_cache()


def test_large_tables_in_a_graph():
    """256 buckets: 131 KB of LDS, asked for at the launch, captured as well."""
    b = R.Buckets.clipped(127, other=True)
    pos, seg = torch.arange(60, dtype=torch.int32).cuda(), (torch.arange(60, dtype=torch.int32) // 25).cuda()
    table, z = normal((256, 128), 1), normal((60, 60, 128), 2)
    d, small = normal((1, 4, 60, 64), 3)[..., :60], normal((256, 4), 4)
    graph = torch.cuda.CUDAGraph()
    call = (b, pos, pos, seg, seg)

    def step():
        return (R.relative_pair(table, *call, base=z), R.relative_pair_backward(z, *call), R.relative_bias(small, *call, base=d),
                R.relative_bias_backward(d, *call))
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        z.copy_(normal((60, 60, 128), 10 + i))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i
