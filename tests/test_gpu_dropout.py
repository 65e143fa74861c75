"""GPU parity of the residual addition with dropout (include/pair_dropout.h) against the oracle: the mask exactly,
values within half a step of the output's type (u = 2^-24 or 2^-8 relative to the result) plus the float32
rounding of 1 / (1 - p), 2^-24 of the dropped term, and of the product in it (the addition is fused)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import dropout as D
from paper_2603_14806_amd import synth
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import errors, host, make_layer, needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(TORCH[dtype]).cuda()


def close(got, ref, term, dtype, what):
    y = host(got)
    assert y.shape == ref.shape
    far = np.abs(y - ref) - (U[dtype] * np.abs(ref) + 2.0 ** -23 * np.abs(term))
    assert (far <= 0).all(), f"{what}: {far.max()} beyond the rounding at {np.unravel_index(far.argmax(), far.shape)}"


SHAPES = [(1, 1, 1), (3, 5, 7), (2, 1, 128), (5, 33, 12), (17, 40, 128), (9, 10, 384), (3, 4, 2056), (64, 3, 8), (2, 700, 30)]


@pytest.mark.parametrize("share", ["none", "rows", "columns"])
@pytest.mark.parametrize("x_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("z_dtype", ["f32", "bf16"])
def test_matches_oracle(x_dtype, z_dtype, share):
    for n, shape in enumerate(SHAPES):
        x, z = normal(shape, n, x_dtype), normal(shape, 50 + n, z_dtype)
        for p, seed, offset in ((0.25, 3 + n, 0), (0.1, (1 << 63) + 12345 * n, (1 << 40) + 7), (0.0, 1, 1)):
            k = oracle.keep(*shape, p, seed, offset, share)
            term = oracle.dropout_add(host(x), None, p, k)
            what = f"{shape} {x_dtype}->{z_dtype} {share} p={p}"
            close(D.dropout_add(x, z, p, seed, offset, share), host(z) + term, term, z_dtype, what)
            close(D.dropout_add(x, None, p, seed, offset, share, out_dtype=z_dtype), term, term, z_dtype, what + " alone")
            back = oracle.dropout_backward(host(z), p, k)
            close(D.dropout_backward(z, p, seed, offset, share, dtype=x_dtype), back, back, x_dtype, what + " backward")


@pytest.mark.parametrize("share", ["none", "rows", "columns"])
def test_tiles_agree_with_the_whole(share):
    """A 2-D grid of tiles, each a view into a larger tensor, gives the whole tensor's result bit for bit."""
    x, z = normal((37, 50, 24), 1, "f32"), normal((37, 50, 24), 2, "bf16")
    whole = D.dropout_add(x, z, 0.3, 9, 4, share)
    back = D.dropout_backward(z, 0.3, 9, 4, share, dtype="f32")
    got, gotb = torch.full_like(z, 7.0), torch.full_like(x, 7.0)
    for r0, r1 in ((0, 16), (16, 37)):
        for c0, c1 in ((0, 21), (21, 22), (22, 50)):
            place = dict(row0=r0, col0=c0, n_cols=50)
            D.dropout_add(x[r0:r1, c0:c1], z[r0:r1, c0:c1], 0.3, 9, 4, share, out=got[r0:r1, c0:c1], **place)
            D.dropout_backward(z[r0:r1, c0:c1], 0.3, 9, 4, share, dtype="f32", out=gotb[r0:r1, c0:c1], **place)
    assert torch.equal(got, whole) and torch.equal(gotb, back)


def test_far_places_and_unaligned_rows():
    """Element numbers past 2^32 blocks, and rows that start off the vector's alignment."""
    place = dict(row0=(1 << 33) + 5, col0=70, n_cols=100)
    for shape, off in (((3, 30, 8), 0), ((3, 30, 8), 3), ((4, 9, 7), 1)):
        flat = normal((shape[0] * (shape[1] * shape[2] + 5) + off,), 3, "bf16")
        x = flat[off:].as_strided(shape, (shape[1] * shape[2] + 5, shape[2], 1), off)
        for share in ("none", "rows", "columns"):
            k = oracle.keep(*shape, 0.4, 11, 0, share, **place)
            term = oracle.dropout_add(host(x), None, 0.4, k)
            close(D.dropout_add(x, None, 0.4, 11, 0, share, **place), term, term, "bf16", f"{shape} {off} {share}")


def test_in_place_and_values_that_are_dropped():
    x, z = normal((20, 30, 16), 1, "bf16"), normal((20, 30, 16), 2, "bf16")
    want = D.dropout_add(x, z, 0.5, 6)
    k = torch.from_numpy(oracle.keep(20, 30, 16, 0.5, 6, 0, "none")).cuda()
    y = torch.where(k, x, torch.full_like(x, float("nan")))    # a dropped value is not looked at
    assert torch.equal(D.dropout_add(y, z, 0.5, 6), want)
    back = D.dropout_backward(z, 0.5, 6)
    a, b, c = z.clone(), x.clone(), z.clone()
    assert D.dropout_add(x, a, 0.5, 6, out=a) is a and torch.equal(a, want)
    assert torch.equal(D.dropout_add(b, z, 0.5, 6, out=b), want)
    assert torch.equal(D.dropout_backward(c, 0.5, 6, out=c), back)


def test_rate_at_size():
    """2^24 values: the share kept within five standard deviations, and different by seed and by offset."""
    one = torch.ones((512, 256, 128), device="cuda")
    m = [D.dropout_add(one, None, 0.25, s, o) > 0 for s, o in ((1, 0), (2, 0), (1, 1))]
    for a in m:
        assert abs(float(a.float().mean()) - 0.75) < 5 * (0.75 * 0.25 / 2 ** 24) ** 0.5
    for a, b in ((0, 1), (0, 2), (1, 2)):                       # independent masks agree on 0.75^2 + 0.25^2
        assert abs(float((m[a] == m[b]).float().mean()) - 0.625) < 5 * (0.625 * 0.375 / 2 ** 24) ** 0.5


def test_streams_graphs_and_refusals():
    x, z = normal((40, 40, 128), 1, "f32"), normal((40, 40, 128), 2, "bf16")
    want = D.dropout_add(x, z, 0.25, 1, 2, "rows")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [D.dropout_add(x, z, 0.25, 1, 2, "rows", stream=t) for t in (s, s.cuda_stream, None)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = D.dropout_add(x, z, 0.25, 1, 2, "rows")
    for i in range(3):
        x.copy_(normal((40, 40, 128), 10 + i, "f32"))
        graph.replay()
        eager = D.dropout_add(x, z, 0.25, 1, 2, "rows")
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
    for bad in (dict(share="row"), dict(seed=-1), dict(seed=1 << 64), dict(offset=-1), dict(out=x), dict(residual=z[:, :, ::2]),
                dict(residual=z[:-1]), dict(residual=z.cpu()), dict(out=torch.empty((40, 40, 160), dtype=torch.bfloat16, device="cuda")[..., :128])):
        with pytest.raises(ValueError):
            D.dropout_add(**{**dict(x=x, residual=z), **bad})
    with pytest.raises(T.TriMulError) as e:
        D.dropout_add(x, z, 1.0)
    assert e.value.code == T.TRI_MUL_EINVAL


@pytest.mark.parametrize("direction", ["outgoing", "incoming"])
def test_triangle_update_with_residual(direction):
    """TriMul.residual and its backward: the layer's own call, dropped and added, against the oracle's update."""
    N, p, seed = 40, 0.25, 5
    layer, W = make_layer("bf16")
    z = synth.pair_tensor(N, dtype="bf16", seed=3, device="cuda")
    mask = synth.token_mask(N, 4, device="cuda")
    k = oracle.keep(N, N, 128, p, seed, 1, "rows")
    got = layer.residual(z, mask, direction, p, seed, 1)
    update = oracle.tri_mul(host(z), host(mask), W, direction)
    ref = oracle.dropout_add(update, host(z), p, k)
    # half a step of bf16 for the sum, and the update's own bar of 5e-3 of its norm
    limit = 2.0 ** -8 * np.linalg.norm(ref) + 5e-3 * np.linalg.norm(update) / (1 - p)
    assert np.linalg.norm(host(got) - ref) <= limit
    dout = normal((N, N, 128), 9, "bf16")
    dz, grads = layer.residual_backward(z, dout, mask, direction, p, seed, 1)
    want = oracle.tri_mul_backward(host(z), host(mask), W, direction, oracle.dropout_backward(host(dout), p, k))
    ref = host(dout) + want["dz"]
    limit = 2.0 ** -8 * np.linalg.norm(ref) + (5e-3 + 2.0 ** -8) * np.linalg.norm(want["dz"])
    say(f"  residual {direction}: dz error {np.linalg.norm(host(dz) - ref):.3e} limit {limit:.3e}")
    assert np.linalg.norm(host(dz) - ref) <= limit
    for n in W:
        mx, rel = errors(host(grads[n]), want[n])
        assert rel <= 5e-3, (n, rel)
    layer.close()
