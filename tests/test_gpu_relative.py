"""GPU parity of the relative position bias by buckets (include/relative_bias.h) against the oracle.

Forward: base and table are added in float32 and rounded once, so within (u + 2^-24) of the result with u half a step of
its type; without a base, and in float32 or of the table's type, the table's values themselves.  Gradient: from whole
numbers of at most 8, whose sums float32 holds, it is equal; from other values each float32 sum of n in sequence is
within n 2^-24 of the sum of magnitudes, and no lane adds more than 128 of them here (the widest call: 1500 rows on 256
lanes' worth of rows and splits), with the sums of lanes in float64 and two roundings at the end."""
import numpy as np
import pytest
import torch

from oracle import relative as O
from paper_2603_14806_amd import attention as A
from paper_2603_14806_amd import relative as R
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import host, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def normal(shape, seed, dtype="f32"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(TORCH[dtype]).cuda()


def whole(shape, seed, dtype="f32"):
    return torch.randint(-8, 9, shape, generator=torch.Generator().manual_seed(seed)).to(TORCH[dtype]).cuda()


def integers(shape, low, high, seed):
    return torch.randint(low, high, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


def padded(t):
    """The same values in rows padded to a multiple of 8, NaN behind them."""
    n = t.shape[-1]
    p = torch.full(tuple(t.shape[:-1]) + (-(-n // 8) * 8,), float("nan"), dtype=t.dtype, device=t.device)
    p[..., :n] = t
    return p[..., :n]


def positions(kind, n, seed):
    if kind == "range":
        return torch.arange(n, dtype=torch.int32).cuda()
    if kind == "any":
        return integers((n,), -60, 60, seed)
    return torch.tensor(([-2 ** 31, 2 ** 31 - 1, 0, -1] * (n // 4 + 1))[:n], dtype=torch.int32).cuda()


PLANS = {"clip": lambda other: R.Buckets.clipped(7, other), "log": lambda other: R.Buckets.logarithmic(12, 40, other=other),
         "past": lambda other: R.Buckets.logarithmic(6, 20, both=False, other=other), "one": lambda other: R.Buckets([0], other),
         "far": lambda other: R.Buckets.logarithmic(240, 4095, other=other), "most": lambda other: R.Buckets.clipped(127, other)}


def where(plan, nq, nk, kind, other, seed):
    b = PLANS[plan](other)
    pq, pk = positions(kind, nq, seed), positions(kind, nk, seed + 1)
    segs = (integers((nq,), 0, 3, seed + 2), integers((nk,), 0, 3, seed + 3)) if other else ()
    rows = O.buckets(b.lut.tolist(), b.rows, *(host(t).astype(np.int64) for t in (pq, pk) + segs))
    return (b, pq, pk) + segs, rows


def near(got, ref, dtype):
    y = host(got)
    assert y.shape == ref.shape and (np.abs(y - ref) <= (U[dtype] + 2.0 ** -24) * np.abs(ref)).all()


CASES = [(1, 1, 1, "clip", "range"), (2, 9, 3, "one", "any"), (64, 64, 4, "clip", "range"), (5, 300, 1, "log", "range"),
         (300, 5, 2, "past", "any"), (33, 77, 12, "log", "extreme"), (70, 530, 9, "far", "range"), (129, 131, 16, "most", "range"),
         (40, 2100, 3, "clip", "any")]


@pytest.mark.parametrize("other", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("table_dtype", ["f32", "bf16"])
def test_bias_matches_oracle(dtype, table_dtype, other):
    for i, (nq, nk, heads, plan, kind) in enumerate(CASES):
        call, rows = where(plan, nq, nk, kind, other, 10 * i)
        table = normal((call[0].rows, heads), i, table_dtype)
        got = R.relative_bias(table, *call, dtype=dtype)
        ref = O.relative_bias(host(table), rows)[None]
        assert got.dtype == TORCH[dtype] and (heads == 1 or got.stride(2) % 8 == 0)
        near(got, ref, dtype)
        if dtype in ("f32", table_dtype):
            assert np.array_equal(host(got), ref)
        base = normal((1, heads, nq, nk), 50 + i, dtype)
        want = O.relative_bias(host(table), rows, host(base)[0])[None]
        aligned = padded(base)
        for b in (aligned, base):                       # rows of any alignment
            near(R.relative_bias(table, *call, base=b), want, dtype)
        assert torch.equal(R.relative_bias(table, *call, base=base[0]), R.relative_bias(table, *call, base=aligned))
        assert R.relative_bias(table, *call, base=aligned, out=aligned) is aligned
        near(aligned, want, dtype)
        dout = padded(whole((1, heads, nq, nk), 90 + i, dtype))
        grad = O.table_gradient(np.moveaxis(host(dout)[0], 0, -1), rows, call[0].rows)
        for d in (dout, dout.contiguous(), dout[0]):
            assert np.array_equal(host(R.relative_bias_backward(d, *call)), grad), (nq, nk, heads, plan, kind)


@pytest.mark.parametrize("other", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("table_dtype", ["f32", "bf16"])
def test_pair_matches_oracle(dtype, table_dtype, other):
    for i, (nq, nk, ch, plan, kind) in enumerate([(1, 1, 1, "clip", "range"), (3, 5, 30, "log", "any"), (20, 70, 128, "clip", "range"), (50, 50, 64, "past", "range"),
                                                  (7, 90, 384, "log", "extreme"), (66, 1, 12, "clip", "any"), (1, 133, 130, "clip", "range"),
                                                  (40, 41, 128, "most", "range"), (9, 33, 100, "far", "range"), (30, 18, 1024, "one", "any"), (2, 2, 2, "clip", "range")]):
        call, rows = where(plan, nq, nk, kind, other, 10 * i)
        table, base = normal((call[0].rows, ch), i, table_dtype), normal((nq, nk, ch), 50 + i, dtype)
        got = R.relative_pair(table, *call, dtype=dtype)
        near(got, O.relative_pair(host(table), rows), dtype)
        want = O.relative_pair(host(table), rows, host(base))
        near(R.relative_pair(table, *call, base=base), want, dtype)
        wide = torch.full((nq, nk * ch + 11), 7.0, dtype=TORCH[dtype], device="cuda")     # rows further apart, off any alignment
        view = wide.as_strided((nq, nk, ch), (nk * ch + 11, ch, 1), 3)
        if nq == 1 or 3 + (nq - 1) * (nk * ch + 11) + nk * ch <= wide.numel():
            view.copy_(base)
            assert R.relative_pair(table, *call, base=view, out=view) is view
            near(view, want, dtype)
            rest = torch.ones_like(wide, dtype=torch.bool)
            rest.as_strided((nq, nk, ch), (nk * ch + 11, ch, 1), 3).fill_(False)
            assert (wide[rest] == 7.0).all()
        d = whole((nq, nk, ch), 90 + i, dtype)
        grad = O.table_gradient(host(d), rows, call[0].rows)
        assert np.array_equal(host(R.relative_pair_backward(d, *call)), grad), (nq, nk, ch, plan, kind)
        view.copy_(d)
        assert np.array_equal(host(R.relative_pair_backward(view, *call)), grad)


def test_entries_and_shared_axes():
    """Positions for each entry, or one for all; bases and gradients shared along batch or heads."""
    b = R.Buckets.clipped(5, other=True)
    n, nq, nk, heads = 3, 20, 45, 4
    table = normal((b.rows, heads), 1)
    pq, pk = integers((n, nq), -10, 10, 2), integers((n, nk), -10, 10, 3)
    sq, sk = integers((n, nq), 0, 2, 4), integers((n, nk), 0, 2, 5)
    for places in ((pq, pk, sq, sk), (pq[0], pk, sq[0], sk[:1]), (pq[1], pk[1], sq[1], sk[1]), (pq[:1], pk[0], sq, sk[1])):
        at = [[host(t if t.dim() == 1 else t[min(e, len(t) - 1)]).astype(np.int64) for t in places] for e in range(n)]
        rows = [O.buckets(b.lut.tolist(), b.rows, *p) for p in at]
        batch = max(t.shape[0] if t.dim() == 2 else 1 for t in places)
        ref = np.stack([O.relative_bias(host(table), r) for r in rows])
        assert np.array_equal(host(R.relative_bias(table, b, *places)), ref[:batch])
        for shape in ((n, heads), (1, heads), (n, 1), (1, 1)):
            base = padded(normal(shape + (nq, nk), 6))
            got = R.relative_bias(table, b, *places, base=base)
            near(got, (host(base) + ref)[:max(batch, shape[0])], "f32")
        d = whole((n, heads, nq, nk), 7)
        want = sum(O.table_gradient(np.moveaxis(host(d)[e], 0, -1), rows[e], b.rows) for e in range(n))
        assert np.array_equal(host(R.relative_bias_backward(d, b, *places)), want)
        one = d[:1, :1].expand(n, heads, nq, nk)
        want = sum(O.table_gradient(np.repeat(host(d)[0, 0][..., None], heads, -1), rows[e], b.rows) for e in range(n))
        assert np.array_equal(host(R.relative_bias_backward(one, b, *places)), want)


@pytest.mark.parametrize("own_places", [False, True])
def test_many_small_entries(own_places):
    """More entries than work-groups, as windows are: several of them to a work-group, and the last with fewer."""
    b = R.Buckets.logarithmic(12, 30, other=True)
    n, nq, nk, heads = 1100, 9, 21, 3
    shape = (n,) if own_places else ()
    places = [integers(shape + (m,), lo, hi, s) for m, lo, hi, s in ((nq, -20, 20, 1), (nk, -20, 20, 2), (nq, 0, 2, 3), (nk, 0, 2, 4))]
    d = padded(whole((n, heads, nq, nk), 5, "bf16"))
    x = host(d)
    at = lambda e: [host(t[e] if own_places else t).astype(np.int64) for t in places]
    want = sum(O.table_gradient(np.moveaxis(x[e], 0, -1), O.buckets(b.lut.tolist(), b.rows, *at(e)), b.rows) for e in range(n))
    assert np.array_equal(host(R.relative_bias_backward(d, b, *places)), want)
    table = normal((b.rows, heads), 6)
    got = R.relative_bias(table, b, *places, base=d, dtype="bf16")
    for e in (0, 511, n - 1):
        near(got[e], x[e] + O.relative_bias(host(table), O.buckets(b.lut.tolist(), b.rows, *at(e))), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_longer_calls(dtype):
    """Splits and tiles: every row of the table within the float32 sums' bound, and the same bits again."""
    call, rows = where("clip", 1500, 700, "range", False, 1)
    d = padded(normal((1, 2, 1500, 700), 2, dtype))
    got = R.relative_bias_backward(d, *call)
    x = np.moveaxis(host(d)[0], 0, -1)
    limit = (128 + 2) * 2.0 ** -24 * O.table_gradient(np.abs(x), rows, call[0].rows)
    assert (np.abs(host(got) - O.table_gradient(x, rows, call[0].rows)) <= limit).all()
    assert torch.equal(got, R.relative_bias_backward(d, *call))
    call, rows = where("log", 600, 350, "range", True, 3)
    z = normal((600, 350, 128), 4, dtype)
    got = R.relative_pair_backward(z, *call)
    limit = (128 + 2) * 2.0 ** -24 * O.table_gradient(np.abs(host(z)), rows, call[0].rows)
    assert (np.abs(host(got) - O.table_gradient(host(z), rows, call[0].rows)) <= limit).all()
    assert torch.equal(got, R.relative_pair_backward(z, *call))
    # differences: the sum of out * dout moves with a table entry as its gradient says (linear, so exactly, in float64)
    table = normal((call[0].rows, 128), 5)
    step = torch.zeros_like(table)
    step[3, 7] = 2.0
    moved = (host(R.relative_pair(table + step, *call)) - host(R.relative_pair(table, *call))) * host(z)
    assert abs(moved.sum() / 2 - host(got)[3, 7]) <= 1e-3 * np.abs(moved).sum() + limit[3, 7]


def test_empty_gradients():
    b, none, some = R.Buckets.clipped(2), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for pq, pk in ((none, some), (some, none)):
        shape = (len(pq), len(pk))
        assert (R.relative_bias_backward(torch.zeros((1, 3) + shape, device="cuda"), b, pq, pk) == 0).all()
        assert (R.relative_pair_backward(torch.zeros(shape + (128,), device="cuda"), b, pq, pk) == 0).all()
        assert R.relative_bias(normal((5, 3), 1), b, pq, pk).shape == (1, 3) + shape
        assert R.relative_pair(normal((5, 3), 1), b, pq, pk).shape == shape + (3,)
    assert (R.relative_bias_backward(torch.zeros((0, 3, 4, 4), device="cuda"), b, some, some) == 0).all()


def test_a_tile_is_the_tile_of_the_whole():
    b = R.Buckets.clipped(6)
    pos = torch.arange(50, dtype=torch.int32).cuda()
    table, z = normal((b.rows, 24), 1), normal((50, 50, 24), 2)
    whole_out = R.relative_pair(table, b, pos, pos, base=z)
    got = torch.empty_like(z)
    grad = 0
    d = whole((50, 50, 24), 3)
    for i in (slice(0, 17), slice(17, 50)):
        for j in (slice(0, 30), slice(30, 50)):
            R.relative_pair(table, b, pos[i], pos[j], base=z[i, j], out=got[i, j])
            grad = grad + R.relative_pair_backward(d[i, j], b, pos[i], pos[j])
    assert torch.equal(got, whole_out) and torch.equal(grad, R.relative_pair_backward(d, b, pos, pos))


def test_attention_with_it_and_its_gradient():
    """The bias as cross_attention takes it (padded rows), and the table's gradient from the attention's dbias."""
    b = R.Buckets.logarithmic(8, 20)
    nq, nk, heads = 30, 45, 4
    g = torch.Generator().manual_seed(1)
    q, dout = (torch.randn((1, nq, heads, 16), generator=g) for _ in range(2))
    k, v = (torch.randn((1, nk, heads, 16), generator=g) for _ in range(2))
    table = torch.randn((b.rows, heads), generator=g)
    pq, pk = torch.arange(nq, dtype=torch.int32) + 5, torch.arange(nk, dtype=torch.int32)
    dev = [t.cuda() for t in (q, k, v)]
    bias = R.relative_bias(table.cuda(), b, pq.cuda(), pk.cuda())
    out, stats = A.cross_attention(*dev, bias, return_stats=True)
    dbias = A.cross_attention_backward(*dev, out, stats, dout.cuda(), bias)[3]
    got = R.relative_bias_backward(dbias, b, pq.cuda(), pk.cuda())
    t = table.double().requires_grad_()
    rows = torch.from_numpy(O.buckets(b.lut.tolist(), b.rows, pq.numpy(), pk.numpy()))
    x = torch.einsum("bihd,bjhd->bhij", q.double(), k.double()) / 4 + t[rows].permute(2, 0, 1)
    o = torch.einsum("bhij,bjhd->bihd", torch.softmax(x, -1), v.double())
    o.backward(dout.double())
    assert np.linalg.norm(host(out) - o.detach().numpy()) <= 1e-5 * np.linalg.norm(o.detach().numpy())
    assert np.linalg.norm(host(got) - t.grad.numpy()) <= 1e-5 * np.linalg.norm(t.grad.numpy())


def test_streams_and_graphs():
    call, _ = where("clip", 90, 70, "range", True, 1)
    table, z = normal((call[0].rows, 128), 2), normal((90, 70, 128), 3, "bf16")
    d = padded(normal((2, 8, 90, 70), 4))
    small = normal((call[0].rows, 8), 5)

    def step(stream=None):
        return (R.relative_pair(table, *call, base=z, stream=stream), R.relative_pair_backward(z, *call, stream=stream),
                R.relative_bias(small, *call, stream=stream), R.relative_bias_backward(d, *call, stream=stream))
    want = step()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for t in (s, s.cuda_stream):
        got = step(t)
        held = [torch.full((1 << 20,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(bool((h == 0xff).all()) for h in held)
    graphs = []
    for _ in range(2):                       # two graphs: a workspace each
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((step(), graph))
    for i in range(3):
        z.copy_(normal((90, 70, 128), 20 + i, "bf16"))
        d.copy_(normal((2, 8, 90, 70), 30 + i))
        for _, graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for got, _ in graphs for x, y in zip(got, want)), i


def test_refusals():
    b, other = R.Buckets.clipped(3), R.Buckets.clipped(3, other=True)
    table, p = normal((7, 4), 1), torch.arange(10, dtype=torch.int32).cuda()
    base = normal((1, 4, 10, 10), 2)
    good = dict(table=table, buckets=b, pos_q=p, pos_k=p)
    for bad in (dict(table=table.cpu()), dict(table=table[:6]), dict(table=table.half()), dict(table=normal((7, 8), 1)[:, ::2]), dict(table=table[None]),
                dict(pos_q=p.long()), dict(pos_q=p.cpu()), dict(pos_k=torch.cat([p, p])[::2]), dict(pos_q=p[None, None]), dict(seg_q=p, seg_k=p), dict(seg_q=p),
                dict(buckets=other), dict(buckets=R.Buckets.clipped(3, device="cpu")), dict(base=base.cpu()), dict(base=base[..., :9]), dict(base=base.bfloat16(), dtype="f32"),
                dict(base=base[:, :3]), dict(base=normal((1, 4, 10, 20), 2)[..., ::2]), dict(out=base[:, :1]), dict(out=base.cpu()), dict(out=base.bfloat16()),
                dict(pos_q=p.expand(2, 10), pos_k=p.expand(3, 10)), dict(pos_q=p.expand(2, 10), base=base.expand(3, 4, 10, 10))):
        with pytest.raises(ValueError):
            R.relative_bias(**{**good, **bad})
    with pytest.raises(T.TriMulError) as e:
        R.relative_bias(table, b, p.expand(2, 10), p, out=base.expand(2, 4, 10, 10))
    assert e.value.code == T.TRI_MUL_EINVAL
    for bad in (base[0, 0], base.cpu(), base.half(), base[..., :9], normal((1, 4, 10, 20), 2)[..., ::2]):
        with pytest.raises(ValueError):
            R.relative_bias_backward(bad, b, p, p)
    z = normal((10, 10, 4), 3)
    for bad in (dict(base=z.cpu()), dict(base=z[:9]), dict(base=z.transpose(0, 1)), dict(out=z.bfloat16()), dict(out=normal((10, 10, 8), 3)[..., ::2]), dict(pos_q=p.expand(2, 10))):
        with pytest.raises(ValueError):
            R.relative_pair(**{**good, **bad})
    for bad in (z.cpu(), z.half(), z[:9], z.transpose(0, 1)):
        with pytest.raises(ValueError):
            R.relative_pair_backward(bad, b, p, p)
