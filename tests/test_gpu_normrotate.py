"""GPU parity of the norms with rotation (include/norm_rotate.h) against the oracle.

Tolerance, with e = 2^-24: u is made of x by a mean and a mean square over at most 256 values (eight in sequence and five
levels of a tree each: 13 e of the mean magnitude and of the square), a reciprocal root (1 ulp, half the square's error)
and three products, so within 24 e of M = r (|x| + mean |x|).  Gain, shift, sine and cosine (1 ulp and 0.4 e of the angle)
and the turn add less than 8 e of what they turn: y within 32 e of the pair's sum of M |gain| + |shift|, plus half a step of
its type.  Backward, with G the pair's sum of |dy| and H = G |gain|: h within 8 e of H, its two means within 13 e more and
what u brings, so dx within 64 e of r (H + mean H + M mean (H M)), plus half a step; dgain and dshift within (64 + rows a
lane adds) e of the sums of G M and G.  (Each constant is the sum of the steps above rounded up to a power of two.)"""
import numpy as np
import pytest
import torch

import oracle
from oracle import normrotate as O
from paper_2603_14806_amd import checkpoint8 as C
from paper_2603_14806_amd import normrotate as N
from paper_2603_14806_amd import trimul as T
from tests.gpu_util import host, needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
E = 2.0 ** -24
EPS = 1e-6


def normal(shape, seed, dtype="f32", scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale + mean).to(TORCH[dtype]).cuda()


def pair_sum(m, rot, pairs):
    """|.| of both members of a pair, in each one's place."""
    s = m.copy()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if pairs == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    s[..., a] = s[..., b] = m[..., a] + m[..., b]
    return s


def sizes(x, norm):
    """M and r."""
    x = host(x)
    r = O.normalise(x, norm, EPS)[1]
    return r * (np.abs(x) + np.abs(x).mean(-1, keepdims=True)), r


def check_forward(y, x, phase, rot, gain, shift, norm, pairs, dtype, what):
    g, s = (None if t is None else host(t) for t in (gain, shift))
    ref = O.norm_rotate(host(x), phase, g, s, norm, pairs, EPS)
    m = sizes(x, norm)[0] * (1 if g is None else np.abs(g)) + (0 if s is None else np.abs(s))
    far = np.abs(host(y) - ref) - 32 * E * pair_sum(m, rot, pairs) - U[dtype] * np.abs(ref)
    assert y.shape == x.shape and (far <= 0).all(), f"{what}: {far.max()} at {np.unravel_index(far.argmax(), far.shape)}"


def check_backward(dx, dgain, dshift, x, dy, phase, rot, gain, norm, pairs, dtype, what, lane_rows=64):
    g = None if gain is None else host(gain)
    ref, rgain, rshift = O.norm_rotate_backward(host(x), host(dy), phase, g, norm, pairs, EPS)
    m, r = sizes(x, norm)
    G = pair_sum(np.abs(host(dy)), rot, pairs)
    H = G * (1 if g is None else np.abs(g))
    limit = 64 * E * r * (H + H.mean(-1, keepdims=True) + m * (H * m).mean(-1, keepdims=True)) + U[dtype] * np.abs(ref)
    far = np.abs(host(dx) - ref) - limit
    assert (far <= 0).all(), f"{what} dx: {far.max()} at {np.unravel_index(far.argmax(), far.shape)}"
    rows = tuple(range(G.ndim - 1))
    for name, got, want, size in (("dgain", dgain, rgain, G * m), ("dshift", dshift, rshift, G)):
        if got is not None:
            far = np.abs(host(got) - want) - (64 + lane_rows) * E * size.sum(rows)
            assert (far <= 0).all(), f"{what} {name}: {far.max()}"


# batch, n, heads of q and of k, d, rot
CASES = [(1, 1, 1, 1, 8, 8), (1, 1, 16, 4, 64, 64), (3, 1, 5, 2, 128, 64), (2, 7, 4, 4, 32, 32), (2, 19, 3, 1, 24, 16), (1, 33, 2, 2, 40, 40),
         (5, 6, 9, 3, 16, 8), (2, 5, 1, 7, 80, 48), (1, 12, 2, 1, 256, 256), (2, 9, 3, 3, 200, 24), (9, 3, 2, 2, 96, 0), (1, 70, 20, 10, 128, 128), (40, 21, 4, 4, 32, 32)]


def places(kind, batch, n, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "shared":
        return torch.arange(n, dtype=torch.int32).cuda()
    if kind == "far":
        return (torch.randint(-2 ** 20, 2 ** 20, (batch, 1), generator=g) + torch.arange(n)).to(torch.int32).cuda()
    return torch.randint(0, 300, (batch, n), generator=g, dtype=torch.int32).cuda()


def setup(case, i, dtype, weights, kind):
    b, n, h, hk, d, rot = case
    mean = 0.7 if i % 2 else 0.0
    qk = normal((b, n, (h + hk) * d), i, dtype, 1.5, mean)
    q, k = qk[..., :h * d].unflatten(-1, (h, d)), qk[..., h * d:].unflatten(-1, (hk, d))
    pos = places(kind, b, n, i) if rot else None
    freqs = N.frequencies(rot) if rot else None
    phase = O.phases(host(pos), host(freqs)) if rot else np.ones((n, 0))
    w = {}
    if weights:
        w = {f"{a}_{x}": normal((d,), 10 * i + j, weights, 0.3, 1.0 if a == "gain" else 0.0)
             for j, (a, x) in enumerate((("gain", "q"), ("gain", "k"), ("shift", "q"), ("shift", "k")))}
        if i % 3 == 2:
            w["shift_q"] = None
    return q, k, pos, freqs, phase, w


@pytest.mark.parametrize("norm,pairs", [("rms", "halves"), ("rms", "adjacent"), ("layer", "halves"), ("layer", "adjacent")])
@pytest.mark.parametrize("dtype,weights,kind", [("f32", "f32", "shared"), ("f32", None, "far"), ("bf16", "bf16", "any"), ("bf16", "f32", "far"), ("bf16", None, "shared")])
def test_matches_oracle(dtype, weights, kind, norm, pairs):
    for i, case in enumerate(CASES):
        q, k, pos, freqs, phase, w = setup(case, i, dtype, weights, kind)
        how = dict(norm=norm, pairs=pairs, eps=EPS, **w)
        rot = case[5]
        yq, yk, cq, ck = N.norm_rotate(q, k, pos, freqs, checkpoint=True, **how)
        plain = N.norm_rotate(q, k, pos, freqs, **how)
        assert torch.equal(plain[0], yq) and torch.equal(plain[1], yk)
        dyq, dyk = normal(q.shape, 100 + i, dtype), normal(k.shape, 200 + i, dtype)
        dq, dk, grads = N.norm_rotate_backward(q, k, dyq, dyk, pos, freqs, **how)
        for x, y, c, dy, dx, name in ((q, yq, cq, dyq, dq, "q"), (k, yk, ck, dyk, dk, "k")):
            what = f"{case} {name}"
            gain, shift = w.get("gain_" + name), w.get("shift_" + name)
            assert (grads["gain_" + name] is None) == (gain is None) and (grads["shift_" + name] is None) == (shift is None)
            check_forward(y, x, phase, rot, gain, shift, norm, pairs, dtype, what)
            check_backward(dx, grads["gain_" + name], grads["shift_" + name], x, dy, phase, rot, gain, norm, pairs, dtype, what)
            codes, powers = oracle.checkpoint8(host(x), case[4])
            assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.powers.cpu().numpy(), powers), what
        # from the checkpoints: what the backward of the values they stand for gives
        a = N.norm_rotate_backward(cq, ck, dyq, dyk, pos, freqs, **how)
        b = N.norm_rotate_backward(cq.unpack(), ck.unpack(), dyq, dyk, pos, freqs, **how)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all((a[2][m] is None and b[2][m] is None) or torch.equal(a[2][m], b[2][m]) for m in b[2])
        # each side by itself
        one = N.norm_rotate(None, k, pos, freqs, **{**how, "gain_q": None, "shift_q": None})
        assert one[0] is None and torch.equal(one[1], yk)
        one = N.norm_rotate_backward(q, None, dyq, None, pos, freqs, **{**how, "gain_k": None, "shift_k": None})
        assert one[1] is None and torch.equal(one[0], dq)


def test_many_rows_and_the_same_bits():
    """More items than waves in the backward (its waves go round), and several entries an item."""
    b, n, h, d = 300, 130, 4, 32
    q, k = normal((b, n, h, d), 1, "bf16"), normal((b, n, h, d), 2, "bf16")
    dyq, dyk = normal((b, n, h, d), 3, "bf16"), normal((b, n, h, d), 4, "bf16")
    gain, shift = normal((d,), 5, mean=1.0), normal((d,), 6)
    freqs = N.frequencies(d)
    for pos in (torch.arange(n, dtype=torch.int32).cuda(), places("any", b, n, 7)):
        phase = O.phases(host(pos), host(freqs))
        how = dict(norm="layer", eps=EPS, gain_q=gain, gain_k=gain, shift_q=shift)
        yq, yk = N.norm_rotate(q, k, pos, freqs, **how)
        check_forward(yq, q, phase, d, gain, shift, "layer", "halves", "bf16", "q")
        check_forward(yk, k, phase, d, gain, None, "layer", "halves", "bf16", "k")
        got = N.norm_rotate_backward(q, k, dyq, dyk, pos, freqs, **how)
        check_backward(got[0], got[2]["gain_q"], got[2]["shift_q"], q, dyq, phase, d, gain, "layer", "halves", "bf16", "q")
        check_backward(got[1], got[2]["gain_k"], None, k, dyk, phase, d, gain, "layer", "halves", "bf16", "k")
        again = N.norm_rotate_backward(q, k, dyq, dyk, pos, freqs, **how)
        assert torch.equal(got[0], again[0]) and torch.equal(got[2]["gain_q"], again[2]["gain_q"]) and torch.equal(got[2]["gain_k"], again[2]["gain_k"])


# batch, n, heads of q and of k, d, rot: enough rows to fill the card's waves, positions of each entry's own, so that a wave takes
# a few heads of several tokens in several steps, the last of them (9, 3, 20, 10 heads) and the last tokens only in part
MANY = [(2, 423, 16, 4, 128, 64), (3, 459, 9, 3, 128, 128), (5, 443, 20, 10, 24, 16), (3, 191, 20, 10, 80, 48), (2, 347, 9, 3, 200, 200),
        (7, 331, 20, 10, 32, 32), (2, 843, 16, 4, 64, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(MANY)))
def test_many_rows_with_positions_of_their_own(i, dtype):
    """Values, codes and gradients against the oracle, and from the codes as from the values they stand for.  A lane adds at
    most 16 rows: eight steps an item, two items a wave."""
    case = MANY[i]
    b, n, h, hk, d, rot = case
    lanes = max(4, 1 << (d // 8 - 1).bit_length())
    assert b * n * (h + hk) >= 4096 * (64 // lanes)
    for j, (norm, pairs) in enumerate((("rms", "adjacent"), ("layer", "halves")) if i % 2 else (("layer", "adjacent"), ("rms", "halves"))):
        q, k, pos, freqs, phase, w = setup(case, i, dtype, "f32" if (i + j) % 2 else dtype, "any")
        how = dict(norm=norm, pairs=pairs, eps=EPS, **w)
        yq, yk, cq, ck = N.norm_rotate(q, k, pos, freqs, checkpoint=True, **how)
        plain = N.norm_rotate(q, k, pos, freqs, **how)
        assert torch.equal(plain[0], yq) and torch.equal(plain[1], yk)
        dyq, dyk = normal(q.shape, 100 + i, dtype), normal(k.shape, 200 + i, dtype)
        dq, dk, grads = N.norm_rotate_backward(q, k, dyq, dyk, pos, freqs, **how)
        for x, y, c, dy, dx, name in ((q, yq, cq, dyq, dq, "q"), (k, yk, ck, dyk, dk, "k")):
            what = f"{case} {norm} {pairs} {name}"
            check_forward(y, x, phase, rot, w["gain_" + name], w["shift_" + name], norm, pairs, dtype, what)
            check_backward(dx, grads["gain_" + name], grads["shift_" + name], x, dy, phase, rot, w["gain_" + name], norm, pairs, dtype, what, 16)
            codes, powers = oracle.checkpoint8(host(x), d)
            assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.powers.cpu().numpy(), powers), what
        a = N.norm_rotate_backward(cq, ck, dyq, dyk, pos, freqs, **how)
        e = N.norm_rotate_backward(cq.unpack(), ck.unpack(), dyq, dyk, pos, freqs, **how)
        assert torch.equal(a[0], e[0]) and torch.equal(a[1], e[1]) and all((a[2][m] is None and e[2][m] is None) or torch.equal(a[2][m], e[2][m]) for m in e[2])
        say(f"  {case} {norm} {pairs}")


def test_far_positions_keep_their_angle():
    """The largest positions at the highest frequency: the float64 angle p f is itself off by 2^-53 of it."""
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 123456789], dtype=torch.int32).cuda()
    x = normal((1, 4, 2, 64), 1)
    y, _ = N.norm_rotate(x, None, pos, N.frequencies(64), eps=EPS)
    phase = O.phases(host(pos), host(N.frequencies(64)))
    ref = O.norm_rotate(host(x), phase, eps=EPS)
    m = pair_sum(sizes(x, "rms")[0], 64, "halves")
    assert (np.abs(host(y) - ref) <= (32 * E + 3 * 2.0 ** 31 * 2.0 ** -53) * m + E * np.abs(ref)).all()


def test_rows_are_independent():
    """Rows of zeros, of equal values, and one that holds NaN or infinity: the others keep their bits."""
    for dtype in ("f32", "bf16"):
        x = normal((2, 5, 3, 40), 1, dtype)
        x[0, 0, 1] = 0
        x[0, 1, 2] = 3.0
        pos, freqs = torch.arange(5, dtype=torch.int32).cuda(), N.frequencies(40)
        dy = normal(x.shape, 2, dtype)
        for norm in ("rms", "layer"):
            y, _ = N.norm_rotate(x, None, pos, freqs, norm=norm)
            dx, _, _ = N.norm_rotate_backward(x, None, dy, None, pos, freqs, norm=norm)
            assert torch.isfinite(y).all() and torch.isfinite(dx).all() and (y[0, 0, 1] == 0).all()
            z, dz = x.clone(), dy.clone()
            z[1, 2, 0, 7], z[1, 3, 1, 3], dz[0, 4, 2, 5] = float("nan"), float("inf"), float("nan")
            y2, _, c, _ = N.norm_rotate(z, None, pos, freqs, norm=norm, checkpoint=True)
            dx2, _, _ = N.norm_rotate_backward(z, None, dz, None, pos, freqs, norm=norm)
            keep = torch.ones((2, 5, 3), dtype=torch.bool, device="cuda")
            keep[1, 2, 0] = keep[1, 3, 1] = False
            assert torch.equal(y[keep], y2[keep]) and torch.isnan(y2[1, 2, 0]).any()
            assert (c.powers[..., 0] == 255).sum() == 2 and (c.powers[..., 0][~keep] == 255).all()
            keep[0, 4, 2] = False
            assert torch.equal(dx[keep], dx2[keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_squares_past_the_range(dtype):
    """Rows whose squares float32 does not hold: u and r are 0, so y is the turned shift, dx 0, and nothing of them is in dgain; the
    others keep their bits."""
    x, dy = normal((2, 5, 3, 40), 1, dtype), normal((2, 5, 3, 40), 2, dtype)
    pos, freqs, gain, shift = torch.arange(5, dtype=torch.int32).cuda(), N.frequencies(40), normal((40,), 3, mean=1.0), normal((40,), 4)
    how = dict(gain_q=gain, shift_q=shift)
    y, _ = N.norm_rotate(x, None, pos, freqs, **how)
    dx, _, _ = N.norm_rotate_backward(x, None, dy, None, pos, freqs, **how)
    z = x.clone()
    z[0, 3, 1] *= 2.0 ** 100
    y2, _, c, _ = N.norm_rotate(z, None, pos, freqs, checkpoint=True, **how)
    dx2, _, grads = N.norm_rotate_backward(z, None, dy, None, pos, freqs, **how)
    keep = torch.ones((2, 5, 3), dtype=torch.bool, device="cuda")
    keep[0, 3, 1] = False
    assert torch.equal(y[keep], y2[keep]) and torch.equal(dx[keep], dx2[keep]) and (dx2[0, 3, 1] == 0).all()
    x[0, 3, 1] = 0
    zero, _ = N.norm_rotate(x, None, pos, freqs, **how)
    assert torch.equal(y2[0, 3, 1], zero[0, 3, 1])
    assert torch.equal(grads["gain_q"], N.norm_rotate_backward(x, None, dy, None, pos, freqs, **how)[2]["gain_q"])
    codes, powers = oracle.checkpoint8(host(z), 40)
    assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.powers.cpu().numpy(), powers)


def test_in_place_strides_and_repeated_inputs():
    pos, freqs = torch.arange(6, dtype=torch.int32).cuda(), N.frequencies(32)
    wide = normal((3, 6, 2, 4, 64), 1, "bf16")
    q, k = wide[:, :, 0, :, :32], wide[:, :, 1, :, 32:]
    want = N.norm_rotate(q.contiguous(), k.contiguous(), pos, freqs)
    dy = normal((3, 6, 4, 32), 2, "bf16")
    back = N.norm_rotate_backward(q.contiguous(), k.contiguous(), dy, dy, pos, freqs)
    got = N.norm_rotate_backward(q, k, dy, dy, pos, freqs)
    assert torch.equal(got[0], back[0]) and torch.equal(got[1], back[1])
    turned = N.norm_rotate(q.transpose(1, 2).contiguous().transpose(1, 2), k, pos, freqs)       # heads before tokens
    assert torch.equal(turned[0], want[0]) and torch.equal(turned[1], want[1])
    before = wide.clone()
    out = N.norm_rotate(q, k, pos, freqs, out_q=q, out_k=k)
    assert out[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(wide[:, :, 0, :, 32:], before[:, :, 0, :, 32:]) and torch.equal(wide[:, :, 1, :, :32], before[:, :, 1, :, :32])
    one = normal((1, 6, 1, 32), 3, "bf16")
    y, _ = N.norm_rotate(one.expand(3, 6, 4, 32), None, pos, freqs)
    assert torch.equal(y, N.norm_rotate(one.expand(3, 6, 4, 32).contiguous(), None, pos, freqs)[0])
    dx, _, _ = N.norm_rotate_backward(one.expand(3, 6, 4, 32), None, one.expand(3, 6, 4, 32), None, pos, freqs)
    assert torch.equal(dx[2, :, 3], dx[0, :, 0])


def test_empty_calls():
    f, w = N.frequencies(16), normal((16,), 1)
    for shape in ((0, 4, 2, 16), (3, 0, 2, 16)):
        x, pos = torch.zeros(shape, device="cuda"), torch.zeros(shape[1], dtype=torch.int32, device="cuda")
        y, _, c, _ = N.norm_rotate(x, None, pos, f, gain_q=w, shift_q=w, checkpoint=True)
        assert y.shape == shape
        for source in (x, c):
            dx, _, grads = N.norm_rotate_backward(source, None, x, None, pos, f, gain_q=w, shift_q=w)
            assert dx.shape == shape and (grads["gain_q"] == 0).all() and (grads["shift_q"] == 0).all()


def test_streams_and_graphs():
    b, n, h, d = 60, 40, 4, 64
    q, k, dy = normal((b, n, h, d), 1, "bf16"), normal((b, n, 2, d), 2, "bf16"), normal((b, n, h, d), 3, "bf16")
    pos, freqs, gain = torch.arange(n, dtype=torch.int32).cuda(), N.frequencies(d), normal((d,), 4, "bf16", 0.2, 1.0)
    how = dict(norm="layer", gain_q=gain, gain_k=gain, shift_q=gain)

    def step(stream=None):
        yq, yk, cq, ck = N.norm_rotate(q, k, pos, freqs, checkpoint=True, stream=stream, **how)
        dq, dk, grads = N.norm_rotate_backward(cq, ck, dy, dy[:, :, :2], pos, freqs, stream=stream, **how)
        return [yq, yk, cq.codes, ck.powers, dq, dk] + [g for g in grads.values() if g is not None]
    want = step()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for t in (s, s.cuda_stream):
        got = step(t)
        held = [torch.full((1 << 20,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(bool((m == 0xff).all()) for m in held)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((step(), graph))
    for i in range(3):
        q.copy_(normal((b, n, h, d), 20 + i, "bf16"))
        for _, graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for got, _ in graphs for x, y in zip(got, want)), i


def test_refusals():
    q, k, pos, f = normal((2, 3, 4, 32), 1), normal((2, 3, 2, 32), 2), torch.arange(3, dtype=torch.int32).cuda(), N.frequencies(32)
    w = normal((32,), 3)
    good = dict(q=q, k=k, positions=pos, freqs=f)
    for bad in (dict(q=q[0]), dict(q=q.half()), dict(k=k.bfloat16()), dict(k=k[:, :2]), dict(k=k[:1]), dict(k=k.cpu()), dict(k=normal((2, 3, 2, 64), 2)[..., ::2]),
                dict(positions=None), dict(positions=pos.long()), dict(positions=pos[:2]), dict(positions=pos.expand(3, 3)), dict(positions=pos.cpu()),
                dict(freqs=f.float()), dict(freqs=f[None]), dict(freqs=f.cpu()), dict(gain_q=w[:16]), dict(gain_q=w.cpu()), dict(gain_q=w, shift_q=w.bfloat16()),
                dict(gain_q=w.double()), dict(norm="batch"), dict(pairs="x"), dict(out_q=k), dict(out_q=q.bfloat16()), dict(k=None, gain_k=w), dict(k=None, out_k=k),
                dict(k=C.pack(k)), dict(q=C.pack(q, 32), k=C.pack(k, 32))):
        with pytest.raises(ValueError):
            N.norm_rotate(**{**good, **bad})
    for bad in (dict(eps=0.0), dict(freqs=N.frequencies(34)[:17]), dict(freqs=N.frequencies(12)), dict(freqs=N.frequencies(64)),
                dict(q=normal((2, 3, 4, 36), 1), k=None, positions=None, freqs=None), dict(q=normal((2 * 3 * 4 * 32 + 1,), 1)[1:].view(2, 3, 4, 32)),
                dict(out_q=normal((1, 3, 4, 32), 1).expand(2, 3, 4, 32))):
        with pytest.raises(T.TriMulError) as e:
            N.norm_rotate(**{**good, **bad})
        assert e.value.code == T.TRI_MUL_EINVAL
    for dq, dk in ((q, None), (q[:1], k), (q.bfloat16(), k), (q.cpu(), k)):
        with pytest.raises(ValueError):
            N.norm_rotate_backward(q, k, dq, dk, pos, f)
    for c in (C.pack(q, 16), C.pack(q.bfloat16(), 32)):
        with pytest.raises(ValueError):
            N.norm_rotate_backward(c, C.pack(k, 32), q, k, pos, f)
