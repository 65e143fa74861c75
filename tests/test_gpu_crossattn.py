"""GPU parity of cross attention (include/cross_attn.h), forward and backward, against the fp64 oracle.

Tolerance, derived.  u is half a step of the storage type relative to the value: 2^-8 for bf16.  The kernels round
in that type the results, the weights P before P V and P^T dout, dS before dS K and dS^T Q; everything else is float32
(D = dout . out is computed from out and what its rounding took from it; the limits allow for the rounded one).  A sum of terms rounded independently
is off by at most u times the root of the sum of their squares (a uniform rounding error has an RMS of u / sqrt(3):
a margin of 1.7).  So with A_i = root sum of squares of dout_i * out_i (D is off by u A_i, the same for all keys):
    out   u (|out| + rss_j P_ij v_j)
    dv    u (|dv| + rss_i P_ij dout_i)
    dq    u (|dq| + scale rss_j dS_ij k_j + scale A_i |sum_j P_ij k_j|)
    dk    u (|dk| + scale rss_i dS_ij q_i + scale rss_i A_i P_ij q_i)
    dbias u (|dbias| + rss over the sharing axes of A_i P_ij)
compared by Frobenius norms.  float32: the same sums with u = 64 * 2^-24 in place of the type's half step, for scores
of magnitude 10 (their rounding, 10 * 2^-24, enters the weights), the exponential's and the sums' own rounding; plus,
as the rounding of a score is not independent of its terms, the sums of the terms' magnitudes at 2^-22."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import attention as A
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import host, needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 64 * 2.0 ** -24, "bf16": 2.0 ** -8}


def normal(shape, g, dtype):
    return torch.randn(shape, generator=g).to(TORCH[dtype])


def make(B, nq, nk, H, Hk, d, dtype, bias=None, mask=None, seed=0):
    g = torch.Generator().manual_seed(seed + 1000 * nq + nk)
    x = dict(q=normal((B, nq, H, d), g, dtype), k=normal((B, nk, Hk, d), g, dtype), v=normal((B, nk, Hk, d), g, dtype),
             dout=normal((B, nq, H, d), g, dtype))
    if bias is not None:
        x["bias"] = normal(bias + (nq, -(-nk // 8) * 8), g, dtype)[..., :nk]
    if mask == "random":
        x["mask"] = (torch.rand((B, nk), generator=g) < 0.7).to(torch.uint8)
    elif mask == "pad":                       # lengths down to none at all in the last entry
        length = torch.tensor([nk - (nk * b) // max(1, B - 1) for b in range(B)])
        x["mask"] = (torch.arange(nk)[None] < length[:, None]).to(torch.uint8)
    elif mask == "shared":
        x["mask"] = (torch.rand((nk,), generator=g) < 0.6)
    return x


def cuda(x):
    """On the device; a bias keeps its padded rows."""
    r = {}
    for n, t in x.items():
        if n == "bias":
            ld = -(-t.shape[-1] // 8) * 8
            full = torch.full(tuple(t.shape[:-1]) + (ld,), float("nan"), dtype=t.dtype)
            full[..., :t.shape[-1]] = t
            t = full.cuda()[..., :t.shape[-1]]
        else:
            t = t.cuda()
        r[n] = t
    return r


def call(x, scale=None, **kw):
    a = {n: x.get(n) for n in ("bias", "mask")}
    out, stats = A.cross_attention(x["q"], x["k"], x["v"], scale=scale, return_stats=True, **a)
    grads = A.cross_attention_backward(x["q"], x["k"], x["v"], out, stats, x["dout"], scale=scale, **a, **kw)
    return dict(zip(("out", "dq", "dk", "dv", "dbias"), (out,) + grads)), stats


def bounds(x, ref, scale, dtype):
    """Root-sum-of-squares and magnitude sums of the docstring, per output."""
    f = {n: host(t) for n, t in x.items()}
    H, Hk, d = f["q"].shape[2], f["k"].shape[2], f["q"].shape[3]
    s = d ** -0.5 if scale is None else scale
    rep = lambda t: np.repeat(np.nan_to_num(t, nan=0, posinf=0, neginf=0).transpose(0, 2, 1, 3), H // Hk, 1)  # noqa: E731
    group = lambda t: t.reshape(t.shape[0], Hk, H // Hk, *t.shape[2:]).sum(2).transpose(0, 2, 1, 3)  # noqa: E731
    q, k, v, g = f["q"].transpose(0, 2, 1, 3), rep(f["k"]), rep(f["v"]), f["dout"].transpose(0, 2, 1, 3)
    P, dS, o = ref["P"], np.abs(ref["dS"]), ref["out"].transpose(0, 2, 1, 3)
    a = np.sqrt((g * o) ** 2).sum(-1, keepdims=True)
    a2 = ((g * o) ** 2).sum(-1, keepdims=True)
    T_ = lambda t: t.transpose(0, 1, 3, 2)  # noqa: E731
    big = P * (np.abs(g) @ T_(np.abs(v)) + a)                     # magnitude of what dS is a difference of
    r = {"out": (np.sqrt(P ** 2 @ v ** 2).transpose(0, 2, 1, 3), (P @ np.abs(v)).transpose(0, 2, 1, 3)),
         "dv": (np.sqrt(group(T_(P ** 2) @ g ** 2)), group(T_(P) @ np.abs(g))),
         "dq": ((s * np.sqrt(dS ** 2 @ k ** 2) + s * np.sqrt(a2) * np.abs(P @ k)).transpose(0, 2, 1, 3), s * (big @ np.abs(k)).transpose(0, 2, 1, 3)),
         "dk": (s * np.sqrt(group(T_(dS ** 2) @ q ** 2)) + s * np.sqrt(group(T_(a2 * P ** 2) @ q ** 2)), s * group(T_(big) @ np.abs(q)))}
    if "bias" in f:
        e, m = a2 * P ** 2, big
        for axis in (0, 1):
            if f["bias"].shape[axis] == 1:
                e, m = e.sum(axis, keepdims=True), m.sum(axis, keepdims=True)
        r["dbias"] = (np.sqrt(e), m)
    out = {}
    for n, (rss, mag) in r.items():
        b = U[dtype] * (np.abs(ref[n]) + rss) + 2.0 ** -22 * mag
        out[n] = float(np.linalg.norm(b))
    return out


def check(got, x, what, dtype, scale=None, rounded=False):
    f = {n: host(t) for n, t in x.items() if n != "mask"}
    mask = None if "mask" not in x else x["mask"].cpu().numpy()
    if mask is not None and mask.ndim == 1:
        mask = mask[None]
    kw = dict(bias=f.get("bias"), mask=mask, scale=scale, rounded=rounded)
    ref = oracle.cross_attention_backward(f["q"], f["k"], f["v"], f["dout"], **kw)
    ref["out"] = oracle.cross_attention(f["q"], f["k"], f["v"], **kw)
    limit = bounds(x, ref, scale, dtype)
    for n, t in got.items():
        if t is None:
            continue
        y = host(t)
        assert y.shape == ref[n].shape, (what, n)
        assert np.isfinite(y).all(), f"{what}: {n} is not finite"
        err, norm = np.linalg.norm(y - ref[n]), np.linalg.norm(ref[n])
        say(f"  {what} {n}: error {err:.2e} of {norm:.2e}, limit {limit[n]:.2e}")
        assert err <= limit[n], f"{what}: {n} is off by {err:.3e}, more than {limit[n]:.3e}"


# one token; one key; odd lengths about the tiles of 32, 64 and 128; splits of few queries over long keys; shared
# key heads; every padded width of d
SHAPES = [(1, 1, 1, 1, 1, 8), (2, 1, 257, 4, 4, 32), (1, 1, 5000, 8, 2, 64), (3, 5, 7, 8, 8, 16), (2, 33, 65, 4, 2, 24),
          (1, 130, 64, 2, 2, 40), (2, 129, 100, 3, 1, 128), (1, 31, 513, 4, 4, 96), (2, 200, 300, 2, 2, 64),
          (1, 3, 2049, 6, 1, 128), (1, 40, 1500, 4, 2, 32), (1, 1100, 40, 4, 2, 64), (1, 1030, 77, 2, 1, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_oracle(shape, dtype):
    B, nq, nk, H, Hk, d = shape
    for bias, mask in ((None, None), ((1, H), "random"), ((B, 1), "pad"), ((B, H), "shared"), ((1, 1), None)):
        what = f"{dtype} {shape} bias={bias} mask={mask}"
        x = cuda(make(B, nq, nk, H, Hk, d, dtype, bias, mask))
        check(call(x)[0], x, what, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(347, 5, 70, 3, 3, 24), (130, 3, 40, 16, 8, 64), (1030, 1, 33, 1, 1, 128), (264, 32, 128, 4, 4, 32)])
def test_many_heads_of_few_queries(shape, dtype):
    """More than 1024 key heads (no multiple of four among them) of 32 columns at most: a wave each."""
    B, nq, nk, H, Hk, d = shape
    for bias, mask in ((None, "pad"), ((B, H), "random"), ((1, 1), None)):
        x = cuda(make(B, nq, nk, H, Hk, d, dtype, bias, mask))
        check(call(x)[0], x, f"{dtype} {shape} bias={bias} mask={mask}", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 130, 1500, 4, 2, 64), (1, 257, 255, 8, 8, 24), (4, 130, 700, 4, 4, 32),
                                   (3, 400, 300, 4, 4, 128), (2, 520, 40, 8, 8, 40)])
def test_small_backward_passes(shape, dtype):
    """Tiles of 32 queries and of 32 keys, on both sides of 256 of them together (one launch or two); without dk
    and dv the same dq and dbias within their error."""
    B, nq, nk, H, Hk, d = shape
    for bias, mask in ((None, None), ((B, H), "random"), ((1, H), "pad")):
        what = f"{dtype} {shape} bias={bias} mask={mask}"
        x = cuda(make(B, nq, nk, H, Hk, d, dtype, bias, mask))
        got, _ = call(x)
        check(got, x, what, dtype)
        out, stats = A.cross_attention(x["q"], x["k"], x["v"], x.get("bias"), x.get("mask"), return_stats=True)
        dq, dk, dv, dbias = A.cross_attention_backward(x["q"], x["k"], x["v"], out, stats, x["dout"], x.get("bias"), x.get("mask"), need_kv=False)
        assert dk is None and dv is None
        check({"dq": dq, "dbias": dbias}, x, what + " alone", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_shared_by_many_entries(dtype):
    """Triangle attention's shape: the rows of a pair tensor as the batch, one bias and its gradient for all (the
    sum over the rows split over work-groups), and the library's own triangle attention on the same inputs."""
    x = cuda(make(50, 70, 70, 4, 4, 32, dtype, (1, 4), "shared"))
    got, _ = call(x)
    check(got, x, f"rows {dtype}", dtype)
    if dtype == "bf16":
        rows = torch.zeros(4, 70, 72, dtype=torch.bfloat16, device="cuda")     # it asks for numbers in the padding
        rows[..., :70] = x["bias"][0]
        tri = T.triangle_attention(x["q"], x["k"], x["v"], rows[..., :70], x["mask"].to(torch.uint8), out_dtype="bf16")
        far = float((tri.float() - got["out"].float()).norm() / got["out"].float().norm())
        assert far <= 2.0 ** -7                                                # two results, each within 2^-8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [3, 140])
def test_rows_left_empty_and_huge_biases(dtype, nq):
    """Entries without a key, queries whose bias is -inf everywhere, and rows of -1e9 or of the type's lowest value
    (which swallow q . k: float32 makes them means over the present keys)."""
    B, nk, H = 3, 150, 2
    x = make(B, nq, nk, H, H, 32, dtype, (B, H), "random")
    x["mask"][1] = 0
    low = torch.finfo(TORCH[dtype]).min
    x["bias"][0, :, 0] = -float("inf")
    x["bias"][0, :, 1] = low
    x["bias"][2, :, 0] = -1e9
    x["bias"][2, 0, 1, ::2] = low
    x["bias"][2, 1, 2, 1:] = -float("inf")
    x["mask"][2, 0] = 1
    x = cuda(x)
    got, stats = call(x)
    check(got, x, f"empty {dtype} nq={nq}", dtype, rounded=True)
    out = got["out"]
    assert not out[1].any() and not out[0, 0].any() and not got["dq"][1].any() and not got["dk"][1].any()
    assert torch.equal(out[2, 2, 1], x["v"][2, 0, 1])          # one key left: its v
    stats = stats[:2 * B * H * nq].view(2, B, H, nq)
    assert torch.isneginf(stats[0, 1]).all() and not stats[1, 1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [2, 70])
def test_absent_keys_may_hold_anything(dtype, nq):
    x = cuda(make(2, nq, 203, 4, 2, 24, dtype, (1, 4), "random"))
    want, _ = call(x)
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = {n: t.clone() for n, t in x.items()}
        gone = x["mask"] == 0
        y["k"][gone] = bad
        y["v"][gone] = bad
        pad = torch.empty(1, 4, nq, 208, dtype=TORCH[dtype], device="cuda")
        pad[..., :203] = x["bias"]
        both = gone.all(0)                                     # the bias is shared: absent in every entry
        pad[..., :203][..., both] = bad
        pad[..., 203:] = bad
        y["bias"] = pad[..., :203]
        got, _ = call(y)
        for n in want:
            a, b = got[n], want[n]
            if n == "dbias":
                assert not a[..., both].any()
            assert torch.equal(a, b), (n, bad)
        gone_kv = got["dk"][gone], got["dv"][gone]
        assert not gone_kv[0].any() and not gone_kv[1].any()


def strided(shape, dtype, kind, g):
    """The same logical tensor in another layout."""
    B, n, H, d = shape
    if kind == "heads first":
        return normal((B, H, n, d), g, dtype).cuda().permute(0, 2, 1, 3)
    if kind == "packed":                                       # one of three interleaved, after a channel offset
        return normal((B, n, 3, H, d + 8), g, dtype).cuda()[:, :, 1, :, 8:]
    if kind == "token first":
        return normal((n, B, H, d), g, dtype).cuda().permute(1, 0, 2, 3)
    return normal((1, n, H, d), g, dtype).cuda().expand(B, n, H, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["heads first", "packed", "token first", "repeated"])
@pytest.mark.parametrize("nq", [9, 75])
def test_strides(dtype, kind, nq):
    g = torch.Generator().manual_seed(5)
    B, nk, H, Hk, d = 2, 90, 4, 2, 40
    x = dict(q=strided((B, nq, H, d), dtype, kind, g), k=strided((B, nk, Hk, d), dtype, kind, g),
             v=strided((B, nk, Hk, d), dtype, kind, g), dout=strided((B, nq, H, d), dtype, kind, g))
    rows = normal((nq, H, B, 96), g, dtype).cuda()             # rows of a bias anywhere
    x["bias"] = rows.permute(2, 1, 0, 3)[..., :nk]
    got, stats = call(x)
    y = {n: t.contiguous() for n, t in x.items() if n != "bias"}
    y["bias"] = x["bias"]
    want, _ = call(y)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    check(got, x, f"{kind} {dtype}", dtype)


def test_axes_of_length_one_have_no_stride():
    """What torch reports as the stride of an axis of length 1 may be anything."""
    x = cuda(make(1, 1, 70, 1, 1, 32, "bf16", (1, 1)))
    want, _ = call(x)
    y = {n: t.as_strided(t.shape, (3, 5 if t.shape[1] == 1 else t.stride(1), 7, 1)) for n, t in x.items() if n != "bias"}
    y["bias"] = x["bias"].as_strided(x["bias"].shape, (1, 1, 72, 1))
    got, _ = call(y)
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_writes_nothing_else(dtype):
    """Outputs inside larger buffers through the C names: the values around them stay."""
    B, nq, nk, H, Hk, d = 2, 37, 45, 4, 2, 24
    x = cuda(make(B, nq, nk, H, Hk, d, dtype, (1, H), "pad"))
    want, stats = call(x)
    w = A.view(x["q"], x["k"], x["v"], x["bias"], x["mask"])

    def inside(n, h):
        full = torch.full((B + 2, n + 3, h + 2, d + 8), 7.0, dtype=TORCH[dtype], device="cuda")
        return full, full[1:B + 1, 1:n + 1, 1:h + 1, 8:] if dtype == "bf16" else full[1:B + 1, 1:n + 1, 1:h + 1, 4:d + 4]

    bufs = {n: inside(nq if n in ("out", "dq") else nk, H if n in ("out", "dq") else Hk) for n in ("out", "dq", "dk", "dv")}
    db = torch.full((1, H, nq, 64), 7.0, dtype=TORCH[dtype], device="cuda")
    ts = {n: A.tensor(x[n]) for n in ("q", "k", "v", "dout")}
    ts.update({n: A.tensor(v) for n, (_, v) in bufs.items()})
    n = A.cross_attn_workspace_size(w)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    A.cross_attn_forward(w, ts["q"], ts["k"], ts["v"], ts["out"], stats, ws, n)
    n = A.cross_attn_backward_workspace_size(w)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    A.cross_attn_backward(w, ts["q"], ts["k"], ts["v"], ts["out"], stats, ts["dout"], ts["dq"], ts["dk"], ts["dv"],
                          A.bias_tensor(db), ws, n)
    for name, (full, v) in bufs.items():
        assert torch.equal(v, want[name]), name
        v.fill_(7.0)
        assert bool((full == 7.0).all()), name
    assert torch.equal(db[..., :nk], want["dbias"]) and bool((db[..., nk:] == 7.0).all())
    # frozen keys: dk and dv are not asked for
    dq, dk, dv, dbias = A.cross_attention_backward(x["q"], x["k"], x["v"], want["out"], stats, x["dout"], x["bias"], x["mask"],
                                                   need_kv=False, need_bias=False)
    assert dk is None and dv is None and dbias is None and torch.equal(dq, want["dq"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_of_zero(dtype):
    for B, nq, nk in ((2, 5, 0), (2, 0, 9), (0, 5, 9), (2, 0, 0)):
        x = cuda(make(B, nq, nk, 4, 2, 32, dtype, (1, 4)))
        got, stats = call(x)
        for n, t in got.items():
            assert not t.any(), (n, B, nq, nk)                 # nothing to attend to or from: zeros throughout
        assert got["dbias"].shape == (1, 4, nq, nk) and got["dk"].shape == x["k"].shape


def test_equal_calls_give_equal_bits_on_any_stream():
    """Two calls at once on two streams, and a third on the default one."""
    x = cuda(make(2, 100, 700, 4, 2, 64, "bf16", (1, 4), "random"))
    few = cuda(make(1, 2, 9000, 4, 2, 64, "bf16", None, "random"))
    want, want_few = call(x)[0], call(few)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    results = []
    for s in streams * 3:
        for y in (x, few):
            out, stats = A.cross_attention(y["q"], y["k"], y["v"], y.get("bias"), y["mask"], return_stats=True, stream=s)
            with torch.cuda.stream(s):
                results.append((y is x, (out,) + A.cross_attention_backward(y["q"], y["k"], y["v"], out, stats, y["dout"], y.get("bias"), y["mask"], stream=s.cuda_stream)))
    torch.cuda.synchronize()
    for is_x, got in results:
        for a, b in zip(got, (want if is_x else want_few).values()):
            assert (a is None and b is None) or torch.equal(a, b)


def test_captured_graphs_replay():
    """A step captured into a graph, replayed with new inputs between eager work, equals the eager call each time."""
    x = cuda(make(2, 70, 900, 4, 2, 32, "bf16", (1, 4), "random"))
    few = cuda(make(1, 1, 6000, 4, 2, 32, "bf16", None, "random"))
    call(x), call(few)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, got_few = call(x)[0], call(few)[0]
    for i in range(4):
        for t in (x, few):
            for n in ("q", "k", "v", "dout"):
                t[n].copy_(torch.randn(t[n].shape, generator=torch.Generator().manual_seed(i)).to(t[n].dtype))
        graph.replay()
        want, want_few = call(x)[0], call(few)[0]
        torch.cuda.synchronize()
        for a, b in ((got, want), (got_few, want_few)):
            for n in a:
                assert a[n] is None or torch.equal(a[n], b[n]), (i, n)


def test_offsets_past_32_bits():
    """One query over 2.2 million keys, 4.5 GB each of k and v (byte and element offsets past 2^32 and 2^31), the
    last keys the ones that matter; and a batch stride as long."""
    nk, H, d = 2200000, 8, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn((1, nk, H, d), generator=g, device="cuda", dtype=torch.bfloat16)
    v = torch.randn((1, nk, H, d), generator=g, device="cuda", dtype=torch.bfloat16)
    q = torch.randn((1, 1, H, d), generator=g, device="cuda", dtype=torch.bfloat16)
    k[:, -3:] = 4 * q
    out = A.cross_attention(q, k, v)
    for h in (0, 7):
        s = (k[0, :, h].float() @ q[0, 0, h].float()).double() / d ** 0.5
        w = torch.softmax(s, 0)
        ref = sum((w[i:i + 200000, None] * v[0, i:i + 200000, h].double()).sum(0) for i in range(0, nk, 200000))
        assert float((out[0, 0, h].double() - ref).norm() / ref.norm()) < 2.0 ** -7, h
    # the same memory as a batch of two long entries
    kk, vv = k.view(2, nk // 2, H, d), v.view(2, nk // 2, H, d)
    q2 = q.expand(2, 1, H, d)
    out2 = A.cross_attention(q2, kk, vv)
    s = (kk[1, :, 3].float() @ q[0, 0, 3].float()).double() / d ** 0.5
    w = torch.softmax(s, 0)
    ref = sum((w[i:i + 200000, None] * vv[1, i:i + 200000, 3].double()).sum(0) for i in range(0, nk // 2, 200000))
    assert float((out2[1, 0, 3].double() - ref).norm() / ref.norm()) < 2.0 ** -7


def on_gpu(q, k, v, dout, scale):
    """float64 reference of one (entry, head) on the device: out, dq, dk, dv."""
    q, k, v, g = (t.double() for t in (q, k, v, dout))
    P = torch.softmax(q @ k.T * scale, -1)
    out = P @ v
    dS = P * (g @ v.T - (g * out).sum(-1, keepdim=True))
    return out, dS @ k * scale, dS.T @ q * scale, P.T @ g


def test_split_gradients_of_wide_heads():
    """2 x 4 key heads of 3000 keys and d = 128: eight waves to 128 keys, and the queries in four splits.  The rounding
    of bf16 results, weights and dS: three errors of RMS 2^-8 / sqrt(3) at most."""
    x = cuda(make(2, 1024, 3000, 16, 4, 128, "bf16"))
    w = A.view(x["q"], x["k"], x["v"])
    rows = 2 * 16 * 1024 * 16                                  # workspace without splits
    assert A.cross_attn_backward_workspace_size(w) > rows + 2 * 2 * 4 * 3000 * 128 * 4
    got, _ = call(x)
    for b, hk in ((0, 0), (1, 3)):
        dk = dv = 0
        for h in range(4 * hk, 4 * hk + 4):
            ref = on_gpu(x["q"][b, :, h], x["k"][b, :, hk], x["v"][b, :, hk], x["dout"][b, :, h], 128 ** -0.5)
            for n, r in (("out", ref[0]), ("dq", ref[1])):
                rel = float((got[n][b, :, h].double() - r).norm() / r.norm())
                say(f"  wide heads {n} b={b} h={h}: {rel:.2e}")
                assert rel <= 2.0 ** -8, (n, rel)
            dk, dv = dk + ref[2], dv + ref[3]
        for n, r in (("dk", dk), ("dv", dv)):
            rel = float((got[n][b, :, hk].double() - r).norm() / r.norm())
            say(f"  wide heads {n} b={b} hk={hk}: {rel:.2e}")
            assert rel <= 2.0 ** -8, (n, rel)


def test_bias_further_apart_than_a_descriptor():
    """The biases of two query heads that share a key head, 2^30 + 64 values apart: the heads are taken singly then,
    with the results of the same biases side by side (each within half a step of bf16)."""
    far = (1 << 30) + 64
    x = cuda(make(1, 50, 60, 2, 1, 32, "bf16", (1, 2), "random"))
    room = torch.empty(far + 50 * 64, dtype=torch.bfloat16, device="cuda")
    bias = room.as_strided((1, 2, 50, 60), (8, far, 64, 1))
    bias.copy_(x["bias"])
    y = dict(x, bias=bias)
    want, got = call(x)[0], call(y)[0]
    for n in ("out", "dq", "dk", "dv", "dbias"):
        assert float((got[n].float() - want[n].float()).norm()) <= 2.0 ** -8 * float(want[n].float().norm()), n
    check(got, x, "far biases", "bf16")


def test_scale_and_python_refusals():
    x = cuda(make(1, 9, 20, 2, 2, 32, "f32"))
    check(call(x, scale=0.3)[0], x, "scale", "f32", scale=0.3)
    q, k, v = x["q"], x["k"], x["v"]
    for bad in (dict(bias=torch.zeros(1, 2, 9, 20, dtype=torch.bfloat16, device="cuda")), dict(bias=torch.zeros(2, 2, 9, 24, device="cuda")[..., :20]),
                dict(bias=torch.zeros(1, 2, 9, 24, device="cuda")), dict(mask=torch.ones(1, 21, dtype=torch.uint8, device="cuda")),
                dict(mask=torch.ones(1, 20, device="cuda")), dict(mask=torch.ones(1, 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            A.cross_attention(q, k, v, **bad)
    with pytest.raises(T.TriMulError) as e:                    # rows 20 values apart
        A.cross_attention(q, k, v, bias=torch.zeros(1, 2, 9, 20, device="cuda"))
    assert e.value.code == T.TRI_MUL_EINVAL
    for a in ((q, k, v[:, :-1]), (q, k.bfloat16(), v), (q[..., ::2], k[..., ::2], v[..., ::2]), (q, k[..., :24], v)):
        with pytest.raises(ValueError):
            A.cross_attention(*a)
    out, stats = A.cross_attention(q, k, v, return_stats=True)
    rep = torch.zeros(1, 1, 9, 24, device="cuda")[..., :20].expand(1, 2, 9, 20)
    with pytest.raises(ValueError, match="length 1"):
        A.cross_attention_backward(q, k, v, out, stats, x["dout"], bias=rep)
    with pytest.raises(ValueError, match="stats"):
        A.cross_attention_backward(q, k, v, out, stats[:1], x["dout"])
