"""GPU parity of activations in 8 bits (include/checkpoint8.h) against the oracle: codes, powers and the values read back
are equal (the scale is a power of two, so each code has one value), and the layer's backward from a checkpoint is the
backward from the tensor it stands for, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import checkpoint8 as C
from paper_2603_14806_amd import synth
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import host, make_layer, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def values(shape, seed, dtype):
    """Groups of very different size, ties among them: whole numbers and halves beside a group's own scale."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-30, 30, shape[:-1] + (1,), generator=g).float())
    half = torch.randint(-256, 256, shape, generator=g).float() / 2
    return torch.where(torch.rand(shape[:-1] + (1,), generator=g) < 0.4, half, x).to(TORCH[dtype])


def same(c, x, group):
    codes, powers = oracle.checkpoint8(host(x), group)
    assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.powers.cpu().numpy(), powers)
    want = oracle.checkpoint8_values(codes, powers, group)
    for dtype in (None, "f32", "bf16"):
        y = c.unpack(dtype)
        assert y.dtype == (x.dtype if dtype is None else TORCH[dtype])
        assert np.array_equal(host(y), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [8, 16, 24, 32, 64, 80, 128, 256])
def test_matches_oracle(dtype, group):
    for i, shape in enumerate([(1, 1), (3, 7), (5, 8), (2, 4, 30), (4, 129), (3, 3, 128), (7, 384), (70, 31, 64), (1, 1000), (2, 520)]):
        x = values(shape, 10 * group + i, dtype).cuda()
        same(C.pack(x, group), x, group)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_apart_rows_and_any_alignment(dtype):
    flat = values((2000,), 3, dtype).cuda()
    for shape, ld, off in (((4, 40), 48, 0), ((4, 40), 41, 0), ((5, 64), 72, 3), ((3, 2, 24), 24, 1), ((2, 30), 32, 8)):
        strides = (ld, 1) if len(shape) == 2 else (2 * ld, ld, 1)
        x = flat.as_strided(shape, strides, off)
        c = C.pack(x, 16)
        same(c, x, 16)
        into = torch.full_like(flat, 7.0)
        view = into.as_strided(shape, strides, off)
        assert c.unpack(out=view) is view
        assert torch.equal(view, c.unpack())
        rest = torch.ones_like(into, dtype=torch.bool)
        rest.as_strided(shape, strides, off).fill_(False)
        assert (into[rest] == 7.0).all()                       # nothing is written between the rows


def test_extremes():
    """Subnormals, the largest values, infinities and NaN, a negative zero, and borders of the scale."""
    big = torch.finfo(torch.float32).max
    rows = [[0.0] * 8, [-0.0] * 8, [2.0 ** -149] * 8, [2.0 ** -133, -2.0 ** -127] * 4, [2.0 ** -121, 1.9921875 * 2.0 ** -121] * 4,
            [1.99 * 2.0 ** -122] * 8, [big, -big] * 4, [float("inf")] + [1.0] * 7, [1.0] * 7 + [float("nan")], [float("-inf"), float("nan")] * 4,
            [1.9921875] + [0.0] * 7, [1.9921874] + [0.5 / 64] * 7, [1.5 / 64, 2.5 / 64, -0.5 / 64, 1.0] * 2]
    x = torch.tensor(rows).cuda()
    c = C.pack(x, 8)
    codes, powers = oracle.checkpoint8(host(x), 8)
    finite = powers[:, 0] != 255
    assert np.array_equal(c.powers.cpu().numpy(), powers) and np.array_equal(c.codes.cpu().numpy()[finite], codes[finite])
    assert np.array_equal(host(c.unpack()), oracle.checkpoint8_values(codes, powers, 8), equal_nan=True)
    # only the group that holds it is lost
    y = torch.randn(2, 96).cuda()
    z = y.clone()
    z[1, 40] = float("nan")
    a, b = C.pack(y).unpack(), C.pack(z).unpack()
    assert torch.isnan(b[1, 32:64]).all() and torch.equal(a[0], b[0]) and torch.equal(a[1, 64:], b[1, 64:]) and torch.equal(a[1, :32], b[1, :32])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_smallest_groups(dtype):
    """Groups whose power is held at 2^-127: codes, powers and values as the oracle's, and errors of at most 2^-128."""
    g = torch.Generator().manual_seed(8)
    top = torch.exp2(torch.rand((300, 1), generator=g, dtype=torch.float64) * 29 - 149)         # up to 2^-120
    x = (top * (2 * torch.rand((300, 40), generator=g, dtype=torch.float64) - 1)).to(TORCH[dtype]).cuda()
    for group in (8, 32):
        same(C.pack(x, group), x, group)
    c = C.pack(x, 8)
    error = np.abs(host(c.unpack()) - host(x)).reshape(300, 5, 8).max(-1)
    held = np.abs(host(x)).reshape(300, 5, 8).max(-1) < 127 * 2.0 ** -128
    assert held.any() and (c.powers.cpu().numpy()[held] == 0).all() and (error[held] <= 2.0 ** -128).all()


def test_large_streams_and_graphs():
    x = values((1 << 14, 1030), 5, "bf16").cuda()
    want = C.pack(x)
    pick = torch.randperm(1 << 14)[:200]
    codes, powers = oracle.checkpoint8(host(x[pick]), 32)
    assert np.array_equal(want.codes[pick].cpu().numpy(), codes) and np.array_equal(want.powers[pick].cpu().numpy(), powers)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for t in (s, s.cuda_stream):
        c = C.pack(x, stream=t)
        y = c.unpack(stream=t)
        torch.cuda.synchronize()
        assert torch.equal(c.codes, want.codes) and torch.equal(y, want.unpack())
    x = values((40, 128), 6, "f32").cuda()
    C.pack(x).unpack()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = C.pack(x).unpack()
    for i in range(3):
        x.copy_(values((40, 128), 20 + i, "f32"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, C.pack(x).unpack())


def test_refusals():
    x = torch.zeros(4, 6, 32, device="cuda")
    for bad in (x[..., ::2], x[:, :4], x.cpu(), x.double(), torch.zeros((), device="cuda")):
        with pytest.raises(ValueError):
            C.pack(bad)
    for group in (0, -8):
        with pytest.raises(ValueError):
            C.pack(x, group)
    for bad, group in ((x, 12), (x, 264), (x[:1, :1].expand(4, 6, 32), 32)):
        with pytest.raises((T.TriMulError, ValueError)):
            C.pack(bad, group)
    c = C.pack(x)
    for bad in (torch.zeros(4, 6, 31, device="cuda"), torch.zeros(4, 6, 32), torch.zeros(4, 6, 32, device="cuda", dtype=torch.float64)):
        with pytest.raises(ValueError):
            c.unpack(out=bad)
    with pytest.raises(ValueError):
        c.unpack("bf16", out=x)
    assert C.pack(x[:0]).unpack().shape == (0, 6, 32) and C.pack(x[..., :0]).unpack().shape == (4, 6, 0)


@pytest.mark.parametrize("direction", ["outgoing", "incoming"])
def test_layer_backward_from_a_checkpoint(direction):
    N = 44
    layer, _ = make_layer("bf16", affine=True)
    z = synth.pair_tensor(N, dtype="bf16", seed=3, device="cuda")
    mask = synth.token_mask(N, 4, device="cuda")
    dout = torch.randn((N, N, 128), generator=torch.Generator().manual_seed(4)).cuda()
    held = C.pack(z)
    stands = held.unpack()
    assert 0 < (stands.float() - z.float()).abs().max() <= z.float().abs().max() / 127
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, s, s.cuda_stream):
        for call, g in ((layer.backward, dout), (layer.residual_backward, dout.to(torch.bfloat16))):
            a, b = call(held, g, mask, direction, stream=stream), call(stands, g, mask, direction, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(a[0], b[0]) and all(torch.equal(a[1][n], b[1][n]) for n in b[1])
    layer.close()


def test_layer_backward_from_a_checkpoint_of_f32_values():
    """A z that was fp32 when it was packed: its values are exact in the layer's bf16.  (A layer in fp32 has no backward, from
    a tensor or from a checkpoint.)"""
    N = 38
    z = synth.pair_tensor(N, dtype="f32", seed=5, device="cuda")
    mask = synth.token_mask(N, 6, device="cuda")
    held = C.pack(z, 64)
    stands = held.unpack("bf16")
    assert held.dtype == torch.float32 and torch.equal(stands.float(), held.unpack())
    for out_dtype in ("f32", "bf16"):
        layer, _ = make_layer("bf16", out_dtype, affine=True)
        dout = torch.randn((N, N, 128), generator=torch.Generator().manual_seed(7)).to(TORCH[out_dtype]).cuda()
        for call, g, more in ((layer.backward, dout, {}), (layer.residual_backward, dout.to(torch.bfloat16), dict(p=0.25, seed=9, share="columns"))):
            a, b = call(held, g, mask, "incoming", **more), call(stands, g, mask, "incoming", **more)
            assert a[0].dtype == torch.bfloat16 and torch.equal(a[0], b[0]) and all(torch.equal(a[1][n], b[1][n]) for n in b[1])
        layer.close()
    layer, _ = make_layer("f32")
    for x in (held, z):
        with pytest.raises(T.TriMulError) as e:
            layer.backward(x, torch.zeros_like(z), mask)
        assert e.value.code == T.TRI_MUL_EUNSUPPORTED
    layer.close()
