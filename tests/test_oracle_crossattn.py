"""Pins of the cross-attention oracle: torch's attention and autograd in float64, differences, and the cases
whose value is known outright (no key, one key, a mask and a bias of -inf, shared heads, huge biases)."""
import numpy as np
import pytest
import torch

import oracle


def inputs(B, nq, nk, H, Hk, d, seed=0):
    r = np.random.default_rng(seed)
    return (r.standard_normal((B, nq, H, d)), r.standard_normal((B, nk, Hk, d)), r.standard_normal((B, nk, Hk, d)),
            r.standard_normal((B, nq, H, d)))


@pytest.mark.parametrize("bias_shape", [None, (1, 1), (2, 1), (1, 6), (2, 6)])
@pytest.mark.parametrize("Hk", [1, 3, 6])
def test_forward_and_gradients_are_torchs(bias_shape, Hk):
    B, nq, nk, H, d = 2, 7, 11, 6, 8
    q, k, v, g = inputs(B, nq, nk, H, Hk, d)
    r = np.random.default_rng(1)
    bias = None if bias_shape is None else r.standard_normal(bias_shape + (nq, nk))
    mask = r.random((B, nk)) < 0.7
    mask[:, 0] = True
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    tb = None if bias is None else torch.tensor(bias, requires_grad=True)
    full = torch.zeros(B, H, nq, nk, dtype=torch.float64) if tb is None else tb.expand(B, H, nq, nk)
    full = full.masked_fill(~torch.tensor(mask)[:, None, None, :], -np.inf)
    rep = [t.permute(0, 2, 1, 3).repeat_interleave(H // Hk, 1) for t in (tk, tv)]
    out = torch.nn.functional.scaled_dot_product_attention(tq.permute(0, 2, 1, 3), *rep, attn_mask=full).permute(0, 2, 1, 3)
    out.backward(torch.tensor(g))
    assert np.allclose(oracle.cross_attention(q, k, v, bias, mask), out.detach().numpy(), rtol=0, atol=1e-13)
    got = oracle.cross_attention_backward(q, k, v, g, bias, mask)
    for name, t in (("dq", tq), ("dk", tk), ("dv", tv), ("dbias", tb)):
        if t is not None:
            assert np.allclose(got[name], t.grad.numpy(), rtol=0, atol=1e-12), name


def test_gradients_are_the_differences():
    q, k, v, g = inputs(1, 3, 5, 2, 1, 8, seed=3)
    bias = np.random.default_rng(4).standard_normal((1, 1, 3, 5))
    mask = np.array([[1, 1, 0, 1, 1]])
    args = dict(q=q, k=k, v=v, bias=bias)
    got = oracle.cross_attention_backward(q, k, v, g, bias, mask, scale=0.7)

    def loss(**changed):
        a = {**args, **changed}
        return float((oracle.cross_attention(a["q"], a["k"], a["v"], a["bias"], mask, 0.7) * g).sum())

    h = 1e-5
    for name, x in args.items():
        for at in list(np.ndindex(x.shape))[::3]:
            step = np.zeros_like(x)
            step[at] = h
            diff = (loss(**{name: x + step}) - loss(**{name: x - step})) / (2 * h)
            assert abs(diff - got["d" + name][at]) < 1e-8, (name, at)


def test_values_known_outright():
    q, k, v, g = inputs(2, 4, 6, 2, 2, 8, seed=5)
    one = np.zeros((2, 6), dtype=np.uint8)
    one[0, 3] = 1                                    # entry 0 has one key, entry 1 none
    k[:, 0], v[:, 1] = np.nan, np.inf                # absent keys may hold anything
    out = oracle.cross_attention(q, k, v, None, one)
    assert np.array_equal(out[0], np.broadcast_to(v[0, 3], out[0].shape)) and not out[1].any()
    got = oracle.cross_attention_backward(q, k, v, g, None, one)
    assert np.allclose(got["dq"], 0, atol=1e-14) and np.allclose(got["dk"], 0, atol=1e-14)
    assert np.array_equal(got["dv"][0, 3], g[0].sum(0)) and not np.delete(got["dv"][0], 3, 0).any() and not got["dv"][1].any()
    q, k, v, g = inputs(1, 4, 6, 2, 2, 8, seed=6)
    bias = np.zeros((1, 1, 4, 6))
    bias[0, 0, 1] = -np.inf                          # a query with no key left
    bias[0, 0, 2] = np.finfo(np.float32).min         # a query whose scores the bias swallows: the plain mean
    out = oracle.cross_attention(q, k, v, bias, None)
    assert not out[0, 1].any() and np.allclose(out[0, 2], v[0].mean(0), atol=1e-14)
    assert oracle.cross_attention(q, k[:, :0], v[:, :0]).any() == False  # noqa: E712


@pytest.mark.parametrize("mistake", ["scale", "mask", "head", "delta", "empty"])
def test_planted_mistakes_are_seen(mistake):
    """Each mistake, planted in a copy of the definition, is further from the oracle than rounding."""
    q, k, v, g = inputs(2, 5, 7, 4, 2, 16, seed=7)
    mask = np.ones((2, 7))
    mask[0, 4:] = 0
    mask[1] = 0
    good = oracle.cross_attention(q, k, v, None, mask)
    if mistake == "scale":
        bad = oracle.cross_attention(q, k, v, None, mask, scale=1.0)
    elif mistake == "mask":
        bad = oracle.cross_attention(q, k, v, None, None)
    elif mistake == "head":                          # key heads taken in turn instead of in groups
        bad = oracle.cross_attention(q[:, :, [0, 2, 1, 3]], k, v, None, mask)[:, :, [0, 2, 1, 3]]
    elif mistake == "empty":                         # a row with no key as a mean of all
        bad = good.copy()
        bad[1] = v[1].mean(0).repeat(2, 0)
    else:                                            # dS without the subtraction of D
        want = oracle.cross_attention_backward(q, k, v, g, None, mask)
        x = want["P"] * np.matmul(g.transpose(0, 2, 1, 3), np.repeat(v.transpose(0, 2, 3, 1), 2, 1))
        assert np.abs(x - want["dS"]).max() > 1e-2
        return
    assert np.abs(bad - good).max() > 1e-2
