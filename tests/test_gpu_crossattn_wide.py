"""GPU parity of cross attention in the forms that large calls take: 128 columns (queries of the heads that share a key
head) to a work-group in the forward and the query pass, 128 keys in the key pass.  They are chosen by the counts
alone, from one tile for each of 256 compute units on; every case here says which forms it has to reach.

Reference in float64 on the device; formulas and limits as in test_gpu_crossattn.py, but by entry and head: the norm of
the error of each (entry, head) against its own limit, so that one wrong row of a tile is seen among many right ones."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import attention as A
from tests.gpu_util import needs_gpu, say
from tests.test_gpu_crossattn import TORCH, U, call, cuda, make, strided

gpu = [pytest.mark.gpu, needs_gpu]


def marked(f):
    for m in gpu:
        f = m(f)
    return f


def tiles(heads, n):
    return heads * -(-n // 128)


def wide_columns(B, nq, nk, H, Hk, d, dtype):
    """Forward and query pass: tiles of 128 columns (else 32, or a wave to each key head)."""
    cols = nq * (H // Hk)
    return tiles(B * Hk, cols) >= 256 and not (cols <= 32 and B * Hk >= 1024)


def wide_keys(B, nq, nk, H, Hk, d, dtype):
    """Key pass: tiles of 128 keys, eight waves each from half as many on in bf16 at d > 64."""
    eight = dtype == "bf16" and d > 64
    return (dtype == "f32" and d > 64) or tiles(B * Hk, nk) >= (128 if eight else 256)


def split(t):
    return t.permute(0, 2, 1, 3).contiguous()


def reference(x, scale=None, rounded=False):
    """(results, limits): float64 tensors of the docstring's formulas; limits without the type's u: (sum of the value
    and the root sums of squares, sum of magnitudes)."""
    f = {n: t.double() for n, t in x.items() if n != "mask"}
    B, nq, H, d = f["q"].shape
    nk, Hk = f["k"].shape[1:3]
    s = d ** -0.5 if scale is None else scale
    m = torch.ones(1, nk, dtype=torch.bool, device=f["q"].device) if "mask" not in x else (x["mask"] != 0).reshape(-1, nk)
    keep = m[:, None, None, :].expand(B, 1, 1, nk)
    q, g = split(f["q"]), split(f["dout"])
    k, v = (split(torch.where(m[:, :, None, None], f[n], 0.0)).repeat_interleave(H // Hk, 1) for n in ("k", "v"))
    T_ = lambda t: t.transpose(2, 3).contiguous()  # noqa: E731
    sc = q @ T_(k) * s
    if "bias" in f:
        sc = sc + torch.where(keep, f["bias"], 0.0)
    if rounded:
        sc = sc.float().double()
    sc = torch.where(keep, sc, -math.inf)
    top = sc.amax(-1, keepdim=True)
    P = torch.exp(sc - torch.where(torch.isfinite(top), top, 0.0))
    total = P.sum(-1, keepdim=True)
    P = P / torch.where(total > 0, total, 1.0)
    o = P @ v
    D = (g * o).sum(-1, keepdim=True)
    dS = P * (g @ T_(v) - D)
    group = lambda t: t.reshape(B, Hk, H // Hk, *t.shape[2:]).sum(2)  # noqa: E731
    a2 = ((g * o) ** 2).sum(-1, keepdim=True)
    big = P * (g.abs() @ T_(v.abs()) + a2.sqrt())
    r = {"out": (o, (P ** 2 @ v ** 2).sqrt(), P @ v.abs()),
         "dq": (dS @ k * s, s * (dS ** 2 @ k ** 2).sqrt() + s * a2.sqrt() * (P @ k).abs(), s * (big @ k.abs())),
         "dk": (group(T_(dS) @ q) * s, s * group(T_(dS ** 2) @ q ** 2).sqrt() + s * group(T_(a2 * P ** 2) @ q ** 2).sqrt(), s * group(T_(big) @ q.abs())),
         "dv": (group(T_(P) @ g), group(T_(P ** 2) @ g ** 2).sqrt(), group(T_(P) @ g.abs()))}
    if "bias" in f:
        b = [dS, a2 * P ** 2, big]
        for axis in (0, 1):
            if f["bias"].shape[axis] == 1:
                b = [t.sum(axis, keepdim=True) for t in b]
        r["dbias"] = (b[0], b[1].sqrt(), b[2])
    return {n: t[0] for n, t in r.items()}, {n: (t[0].abs() + t[1], t[2]) for n, t in r.items()}


def check(got, x, what, dtype, rounded=False):
    want, limits = reference(x, rounded=rounded)
    for n, ref in want.items():
        y = got[n].double()
        y = y if n == "dbias" else y.permute(0, 2, 1, 3)
        assert y.shape == ref.shape, (what, n)
        assert bool(torch.isfinite(y).all()), f"{what}: {n} is not finite"
        err = (y - ref).flatten(2).norm(dim=-1)
        limit = (U[dtype] * limits[n][0] + 2.0 ** -22 * limits[n][1]).flatten(2).norm(dim=-1)
        worst = float((err / limit.clamp(min=1e-300)).max()) if err.numel() else 0.0
        say(f"  {what} {n}: worst (entry, head) at {worst:.2f} of its limit")
        assert bool((err <= limit).all()), f"{what}: {n} at {worst:.3f} of its limit"


def test_reference_is_the_oracles():
    for bias, mask in ((None, None), ((1, 4), "random"), ((3, 1), "pad"), ((3, 4), "shared")):
        x = make(3, 7, 20, 4, 2, 16, "f32", bias, mask)
        f = {n: t.double().numpy() for n, t in x.items() if n != "mask"}
        m = None if "mask" not in x else x["mask"].numpy().reshape(-1, 20)
        ref = oracle.cross_attention_backward(f["q"], f["k"], f["v"], f["dout"], f.get("bias"), m)
        ref["out"] = oracle.cross_attention(f["q"], f["k"], f["v"], f.get("bias"), m)
        got, _ = reference(x)
        for n, t in got.items():
            t = t if n == "dbias" else t.permute(0, 2, 1, 3)
            assert np.abs(t.numpy() - ref[n]).max() < 1e-12, n


# ragged in every axis; a partial last tile of columns with waves that have none; one live wave to a tile; every width
SHAPES = [(70, 150, 203, 4, 4, 32), (40, 300, 130, 8, 4, 64), (33, 129, 70, 8, 8, 24), (20, 140, 333, 16, 16, 40),
          (36, 130, 150, 4, 4, 96), (64, 135, 100, 4, 2, 128), (300, 5, 70, 1, 1, 32), (130, 3, 300, 8, 2, 64),
          (1, 8300, 150, 8, 4, 16), (2, 1030, 2500, 16, 16, 32)]


@marked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_float64(shape, dtype):
    B, nq, nk, H, Hk, d = shape
    assert wide_columns(*shape, dtype)
    assert wide_keys(*shape, dtype) or shape == (1, 8300, 150, 8, 4, 16)
    for bias, mask in ((None, None), (None, "pad"), ((1, H), "random"), ((B, H), "pad"), ((B, 1), "shared"), ((1, 1), None)):
        x = cuda(make(B, nq, nk, H, Hk, d, dtype, bias, mask))
        check(call(x)[0], x, f"{dtype} {shape} bias={bias} mask={mask}", dtype)


@marked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("own", [True, False])
def test_rows_left_empty_and_huge_biases(own, d, dtype):
    """Entries without a key, queries whose bias is -inf everywhere, rows of -1e9 or of the type's lowest value; the
    bias an entry's own (its gradient from the query pass) or shared by all (from a pass of its own)."""
    B, nq, nk, H = 70, 140, 150, 4
    assert wide_columns(B, nq, nk, H, H, d, dtype) and wide_keys(B, nq, nk, H, H, d, dtype)
    x = make(B, nq, nk, H, H, d, dtype, (B if own else 1, H), "random")
    x["mask"][1] = 0
    x["mask"][2, :64] = 0                                      # a whole chunk of keys
    x["mask"][3, :149] = 0
    x["mask"][3, 149] = 1
    low, b = torch.finfo(TORCH[dtype]).min, x["bias"]
    for i in (0, 37, 139):                                     # rows of the first and of the last, partial tile
        b[0, :, i] = -float("inf")
        b[-1, :, i + 1 if i < 139 else 1] = low
    b[0, :, 70] = -1e9
    b[0, 0, 71, ::2] = low
    b[0, 1, 72, 1:] = -float("inf")
    b[0, 2, 73, :64] = -float("inf")
    if dtype == "bf16":                                        # large, and the differences still matter: a float32 score
        b[0, 3, 74] += 2000.0                                  # there has steps of 2^-13, far below bf16's limit
    x["mask"][0, 0] = 1
    x = cuda(x)
    got, stats = call(x)
    check(got, x, f"empty {dtype} d={d} own={own}", dtype, rounded=True)
    assert not got["out"][1].any() and not got["dq"][1].any() and not got["dk"][1].any() and not got["dv"][1].any()
    assert not got["out"][0, [0, 37, 139]].any() and not got["dq"][0, [0, 37, 139]].any()
    assert torch.equal(got["out"][0, 72, 1], x["v"][0, 0, 1])  # one key left: its v
    stats = stats[:2 * B * H * nq].view(2, B, H, nq)
    assert torch.isneginf(stats[0, 1]).all() and not stats[1, 1].any()


@marked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(70, 140, 203, 4, 4, 32), (64, 135, 203, 4, 2, 128), (40, 300, 130, 8, 4, 64)])
def test_absent_keys_may_hold_anything(shape, dtype):
    B, nq, nk, H, Hk, d = shape
    assert wide_columns(*shape, dtype) and wide_keys(*shape, dtype)
    x = make(B, nq, nk, H, Hk, d, dtype, (1, H), "random")
    x["mask"][:, 64:128] = 0                                   # a chunk, and single keys, that no entry has
    x["mask"][:, 5] = 0
    x = cuda(x)
    want, _ = call(x)
    gone = x["mask"] == 0
    both = gone.all(0)
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = {n: t.clone() for n, t in x.items()}
        y["k"][gone] = bad
        y["v"][gone] = bad
        pad = torch.full((1, H, nq, -(-nk // 8) * 8), bad, dtype=TORCH[dtype], device="cuda")
        pad[..., :nk] = x["bias"]
        pad[..., :nk][..., both] = bad
        y["bias"] = pad[..., :nk]
        got, _ = call(y)
        for n in want:
            assert torch.equal(got[n], want[n]), (n, bad)
        assert not got["dk"][gone].any() and not got["dv"][gone].any() and not got["dbias"][..., both].any()


@marked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["heads first", "packed", "token first", "repeated"])
def test_strides(kind, dtype):
    g = torch.Generator().manual_seed(5)
    B, nq, nk, H, Hk, d = 80, 75, 200, 4, 2, 40
    assert wide_columns(B, nq, nk, H, Hk, d, dtype) and wide_keys(B, nq, nk, H, Hk, d, dtype)
    x = dict(q=strided((B, nq, H, d), dtype, kind, g), k=strided((B, nk, Hk, d), dtype, kind, g),
             v=strided((B, nk, Hk, d), dtype, kind, g), dout=strided((B, nq, H, d), dtype, kind, g))
    x["bias"] = torch.randn((nq, H, B, 208), generator=g).to(TORCH[dtype]).cuda().permute(2, 1, 0, 3)[..., :nk]
    got, _ = call(x)
    y = {n: t.contiguous() for n, t in x.items() if n != "bias"}
    y["bias"] = x["bias"]
    want, _ = call(y)
    assert all(torch.equal(got[n], want[n]) for n in want)
    check(got, x, f"{kind} {dtype}", dtype)


@marked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("own", [True, False])
def test_writes_nothing_else(own, dtype):
    """Outputs inside larger buffers through the C names: the values around them stay."""
    B, nq, nk, H, Hk, d = 70, 150, 205, 4, 4, 24
    assert wide_columns(B, nq, nk, H, Hk, d, dtype) and wide_keys(B, nq, nk, H, Hk, d, dtype)
    x = cuda(make(B, nq, nk, H, Hk, d, dtype, (B if own else 1, H), "pad"))
    want, stats = call(x)
    w = A.view(x["q"], x["k"], x["v"], x["bias"], x["mask"])

    def inside(n, h):
        full = torch.full((B + 2, n + 3, h + 2, d + 8), 7.0, dtype=TORCH[dtype], device="cuda")
        return full, full[1:B + 1, 1:n + 1, 1:h + 1, 8:] if dtype == "bf16" else full[1:B + 1, 1:n + 1, 1:h + 1, 4:d + 4]

    bufs = {n: inside(nq if n in ("out", "dq") else nk, H if n in ("out", "dq") else Hk) for n in ("out", "dq", "dk", "dv")}
    db = torch.full((B if own else 1, H, nq, 216), 7.0, dtype=TORCH[dtype], device="cuda")
    again = torch.full((stats.numel() + 64,), 7.0, device="cuda")
    ts = {n: A.tensor(x[n]) for n in ("q", "k", "v", "dout")}
    ts.update({n: A.tensor(v) for n, (_, v) in bufs.items()})
    n = A.cross_attn_workspace_size(w)
    assert n == 0
    A.cross_attn_forward(w, ts["q"], ts["k"], ts["v"], ts["out"], again, None, 0)
    n = A.cross_attn_backward_workspace_size(w)
    ws = torch.full((n + 256,), 7, dtype=torch.uint8, device="cuda")
    A.cross_attn_backward(w, ts["q"], ts["k"], ts["v"], ts["out"], again, ts["dout"], ts["dq"], ts["dk"], ts["dv"],
                          A.bias_tensor(db), ws, n)
    for name, (full, v) in bufs.items():
        assert torch.equal(v, want[name]), name
        v.fill_(7.0)
        assert bool((full == 7.0).all()), name
    assert torch.equal(db[..., :nk], want["dbias"]) and bool((db[..., nk:] == 7.0).all())
    assert bool((ws[n:] == 7).all()) and bool((again[stats.numel():] == 7.0).all())


@marked
def test_streams_and_graphs():
    """Calls at once on two streams, and a captured step replayed with new inputs, give the bits of calls alone."""
    shape = (70, 140, 200, 4, 4, 32)
    assert wide_columns(*shape, "bf16") and wide_keys(*shape, "bf16")
    x = cuda(make(*shape, "bf16", (1, 4), "random"))
    want = call(x)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    results = []
    for s in streams * 2:
        with torch.cuda.stream(s):
            results.append(call(x)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(r[n], want[n]) for r in results for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(x)[0]
    for i in range(3):
        for n in ("q", "k", "v", "dout"):
            x[n].copy_(torch.randn(x[n].shape, generator=torch.Generator().manual_seed(i)).to(x[n].dtype))
        graph.replay()
        want = call(x)[0]
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), i
