"""What bf16's rounding takes from out is kept for the backward: out + rest is the float32 result, and D = dout . out is
made of both.

Inputs for which nothing else is rounded on the way to it: q = 0 (or k = 0), so every weight is 1 / nk and enters
its product as 1, and values that are nearly the same for all keys, v_j = c + w_j / 64, so that dS_ij = (dout_i . v_j -
D_i) / nk is small against D.  With u = 2^-8, half a step of bf16, and A_i the root sum of squares of dout_i * out_i:

  out + rest   rest is within u |out| and rounded by u of itself: u^2 |out|; the float32 sums: a margin of 2^-20
  D            eps_i = u^2 A_i + 2^-20 sum |dout_i out_i|, against u A_i from out alone
  dq           u (|dq| + scale rss_j dS_ij k_j) + scale eps_i |sum_j P_ij k_j|     (dS enters its product as bf16)
  dk           u (|dk| + scale rss_i dS_ij q_i) + scale rss_i eps_i P_ij q_i
  dbias        u |dbias| + rss of eps_i P_ij over those who share the bias
  each plus 2^-22 of the sum of its terms' magnitudes, compared by Frobenius norms.

That these limits tell the two apart is checked without the library: D made of the rounded out is far outside them."""
import numpy as np
import pytest
import torch

from paper_2603_14806_amd import attention as A
from tests.gpu_util import host, needs_gpu, say

u = 2.0 ** -8

# (form, B, nq, nk, H, Hk, d)
FORMS = [("side by side", 1, 100, 5, 4, 4, 32), ("32 columns", 8, 200, 8, 8, 8, 24), ("a wave a head", 300, 3, 6, 4, 4, 32),
         ("128 columns", 70, 150, 5, 4, 4, 64), ("128 columns, wide heads", 70, 140, 7, 4, 4, 128), ("side by side, grouped", 2, 30, 3, 6, 2, 40),
         ("splits joined", 1, 2, 4000, 4, 4, 64), ("splits joined, grouped", 2, 1, 3000, 8, 2, 128)]


def inputs(B, nq, nk, H, Hk, d, zero, shared):
    g = torch.Generator().manual_seed(1000 * nq + nk)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x = dict(q=r(B, nq, H, d), k=r(B, nk, Hk, d), v=r(B, 1, Hk, d) + r(B, nk, Hk, d) / 64, dout=r(B, nq, H, d))
    x[zero].zero_()
    x = {n: t.to(torch.bfloat16) for n, t in x.items()}
    x["bias"] = torch.zeros(1 if shared else B, H, nq, -(-nk // 8) * 8, dtype=torch.bfloat16)[..., :nk]
    return x


def rounded(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def results(x, rest=True):
    """(values, limits by Frobenius norm), numpy float64; without rest: D from the rounded out."""
    f = {n: host(t) for n, t in x.items()}
    B, nq, H, d = f["q"].shape
    nk, Hk = f["k"].shape[1:3]
    s, n = d ** -0.5, H // Hk
    head = lambda t: t.transpose(0, 2, 1, 3)  # noqa: E731
    group = lambda t: t.reshape(B, Hk, n, nk, d).sum(2)  # noqa: E731
    q, g, k, v = head(f["q"]), head(f["dout"]), np.repeat(head(f["k"]), n, 1), np.repeat(head(f["v"]), n, 1)
    P = np.full((B, H, nq, nk), 1.0 / nk)
    out = P @ v
    D = (g * (out if rest else rounded(out))).sum(-1, keepdims=True)
    dS = P * (g @ v.transpose(0, 1, 3, 2) - D)
    eps = u * u * np.sqrt(((g * out) ** 2).sum(-1, keepdims=True)) + 2.0 ** -20 * np.abs(g * out).sum(-1, keepdims=True)
    big = P * (np.abs(g) @ np.abs(v).transpose(0, 1, 3, 2) + np.abs(g * out).sum(-1, keepdims=True))
    t = lambda a: a.transpose(0, 1, 3, 2)  # noqa: E731
    w, e, m = dS, (eps * P) ** 2, big
    for axis in (0, 1):
        if f["bias"].shape[axis] == 1:
            w, e, m = (a.sum(axis, keepdims=True) for a in (w, e, m))
    r = {"dq": (head(s * dS @ k), head(s * np.sqrt(dS ** 2 @ k ** 2)), head(s * eps * np.abs(P @ k)), head(s * big @ np.abs(k))),
         "dk": (head(s * group(t(dS) @ q)), head(s * np.sqrt(group(t(dS) ** 2 @ q ** 2))),
                head(s * np.sqrt(group(t((eps * P) ** 2) @ q ** 2))), head(s * group(t(big) @ np.abs(q)))),
         "dbias": (w, np.zeros_like(w), np.sqrt(e), m)}
    limits = {n: float(np.linalg.norm(u * (np.abs(a) + b) + c + 2.0 ** -22 * m)) for n, (a, b, c, m) in r.items()}
    return dict({n: a[0] for n, a in r.items()}, out=head(out)), limits


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("form", FORMS[:1] + FORMS[1:2] + FORMS[5:], ids=lambda f: f[0])
def test_the_limits_tell_a_rounded_out_apart(form, shared):
    for zero, n in (("q", "dq"), ("k", "dk")):
        x = inputs(*form[1:], zero, shared)
        (want, limits), (off, _) = results(x), results(x, rest=False)
        for name in (n, "dbias"):
            assert np.linalg.norm(off[name] - want[name]) > 1.5 * limits[name], name


@pytest.mark.gpu
@needs_gpu
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0])
def test_what_rounding_took_is_kept(form, shared):
    B, nq, nk, H, Hk, d = form[1:]
    for zero, n in (("q", "dq"), ("k", "dk")):
        x = inputs(*form[1:], zero, shared)
        want, limits = results(x)
        y = {m: t.cuda() for m, t in x.items()}
        pad = torch.zeros(x["bias"].shape[:3] + (-(-nk // 8) * 8,), dtype=torch.bfloat16, device="cuda")
        y["bias"] = pad[..., :nk]
        out, stats = A.cross_attention(y["q"], y["k"], y["v"], y["bias"], return_stats=True)
        first = -(-8 * B * H * nq // 256) * 64                  # floats before the rest: maxima and sums, a multiple of 256 bytes
        rest = stats[first:].view(torch.bfloat16)[:B * H * nq * d].view(B, H, nq, d).permute(0, 2, 1, 3)
        whole, v = host(out) + host(rest), np.abs(host(x["v"])).max()
        far = np.abs(whole - want["out"]) - (u * u * np.abs(want["out"]) + 2.0 ** -20 * v)
        say(f"  {form[0]} zero {zero}: out + rest within {np.abs(whole - want['out']).max():.1e}")
        assert (far <= 0).all(), far.max()
        got = dict(zip(("dq", "dk", "dv", "dbias"), A.cross_attention_backward(y["q"], y["k"], y["v"], out, stats, y["dout"], y["bias"])))
        for name in (n, "dbias"):
            err = float(np.linalg.norm(host(got[name]) - want[name]))
            say(f"  {form[0]} shared={shared} {name}: error {err:.2e}, limit {limits[name]:.2e}")
            assert err <= limits[name], (name, err, limits[name])
