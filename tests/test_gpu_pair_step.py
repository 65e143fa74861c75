"""A training step of two pair-stack blocks, as a program on the library writes it: z1 = z + dropout(triangle update),
z2 = z1 + dropout(triangle attention of z1, by cross_attention with the rows as the batch and one bias for all), and
the gradients of z and of every weight through both, against float64 autograd of the same formulas on the CPU.

Tolerance: bf16 values are rounded once each on the way -- z1, the projections of z1, the attention's weights and
its result, z2: five roundings of half a step, 2^-8, each at most as large in the result as the tensor it is made
from here (weights of variance 1 / 128, gains near 1), so 5 * 2^-8 of the norm forward; backward the gradients of the
same five, dS and du as well: 12 * 2^-8.  (The mask is exact: one wrong element would be far outside.)"""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import attention, dropout, synth
from tests.gpu_util import host, make_layer, needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

N, H, C, P = 28, 4, 128, 0.25


def layer_norm(x, w, b):
    return torch.nn.functional.layer_norm(x, (C,), w, b, oracle.EPS)


def update(z, m, W):
    x = layer_norm(z, W["ln_in_w"], W["ln_in_b"])
    pair = (m[:, None] * m[None])[..., None]
    a = pair * torch.sigmoid(x @ W["w_ga"].T) * (x @ W["w_a"].T)
    b = pair * torch.sigmoid(x @ W["w_gb"].T) * (x @ W["w_b"].T)
    c = torch.einsum("ikc,jkc->ijc", a, b)
    return pair * torch.sigmoid(x @ W["w_g"].T) * (layer_norm(c, W["ln_out_w"], W["ln_out_b"]) @ W["w_o"].T)


def heads(t):
    return t.reshape(N, N, H, 32)


def reference(z, m, W, A, keep1, keep2, dout):
    """float64: (z2, gradients of z, W, A)."""
    z = z.clone().requires_grad_()
    W = {k: v.clone().requires_grad_() for k, v in W.items()}
    A = {k: v.clone().requires_grad_() for k, v in A.items()}
    z1 = z + torch.where(keep1, update(z, m, W) / (1 - P), 0.0)
    q, k, v = (heads(z1 @ A[n].T) for n in ("q", "k", "v"))
    bias = (z1 @ A["b"].T).permute(2, 0, 1)                                 # [H][j][k]
    s = torch.einsum("ijhd,ikhd->ihjk", q, k) / 32 ** 0.5 + bias
    s = s.masked_fill(m[None, None, None, :] == 0, -np.inf)
    o = torch.einsum("ihjk,ikhd->ijhd", torch.softmax(s, -1), v).reshape(N, N, C)
    z2 = z1 + torch.where(keep2, o / (1 - P), 0.0)
    z2.backward(dout)
    return z2.detach(), dict(z=z.grad, **{k: v.grad for k, v in W.items()}, **{"attn_" + k: v.grad for k, v in A.items()})


def step(layer, z, m, A, dout, seed):
    """The step on the library; the projections are torch products in float32."""
    f = {k: v.float() for k, v in A.items()}
    z1 = layer.residual(z, m, "outgoing", P, seed, 0, share="rows")
    x = z1.float().reshape(N * N, C)
    q, k, v = (heads((x @ f[n].T).to(torch.bfloat16)) for n in ("q", "k", "v"))
    bias = torch.zeros(H, N, -(-N // 8) * 8, dtype=torch.bfloat16, device="cuda")
    bias[..., :N] = (x @ f["b"].T).reshape(N, N, H).permute(2, 0, 1).to(torch.bfloat16)
    bias = bias[..., :N]
    o, stats = attention.cross_attention(q, k, v, bias, m, return_stats=True)
    z2 = dropout.dropout_add(o.reshape(N, N, C), z1, P, seed, 1, share="columns")
    do = dropout.dropout_backward(dout, P, seed, 1, share="columns")
    dq, dk, dv, db = attention.cross_attention_backward(q, k, v, o, stats, heads(do), bias, m)
    g = {n: t.float().reshape(N * N, C) for n, t in (("q", dq), ("k", dk), ("v", dv))}
    g["b"] = db.float().permute(1, 2, 0).reshape(N * N, H)
    dA = {"attn_" + n: g[n].T @ x for n in g}
    dz1 = (dout.float().reshape(N * N, C) + sum(g[n] @ f[n] for n in g)).to(torch.bfloat16).reshape(N, N, C)
    dz, dW = layer.residual_backward(z, dz1, m, "outgoing", P, seed, 0, share="rows")
    return z2, dict(z=dz, **dW, **dA)


def test_two_blocks_forward_and_backward():
    layer, W = make_layer("bf16", affine=True)
    g = torch.Generator().manual_seed(12)
    A = {n: (torch.randn((C, C), generator=g) / C ** 0.5).to(torch.bfloat16) for n in ("q", "k", "v")}
    A["b"] = (torch.randn((H, C), generator=g) / C ** 0.5).to(torch.bfloat16)
    z = synth.pair_tensor(N, dtype="bf16", seed=4)
    m = synth.token_mask(N, 3)
    dout = torch.randn((N, N, C), generator=g).to(torch.bfloat16)
    seed = 2024
    keep1, keep2 = (torch.from_numpy(oracle.keep(N, N, C, P, seed, o, s)) for o, s in ((0, "rows"), (1, "columns")))
    Wd = {k: torch.from_numpy(v) for k, v in W.items()}
    assert np.abs(update(z.double(), m.double(), Wd).numpy() - oracle.tri_mul(host(z), host(m), W, "outgoing")).max() < 1e-10
    want, grads = reference(z.double(), m.double(), Wd, {k: v.double() for k, v in A.items()}, keep1, keep2, dout.double())
    dev = {k: v.cuda() for k, v in A.items()}
    got, got_grads = step(layer, z.cuda(), m.cuda(), dev, dout.cuda(), seed)
    rel = float(torch.linalg.norm(got.double().cpu() - want) / torch.linalg.norm(want))
    say(f"  two blocks z2: {rel:.2e}")
    assert rel <= 5 * 2.0 ** -8
    assert set(got_grads) == set(grads)
    for n, r in grads.items():
        rel = float(torch.linalg.norm(got_grads[n].double().cpu() - r) / torch.linalg.norm(r))
        say(f"  two blocks d{n}: {rel:.2e}")
        assert rel <= 12 * 2.0 ** -8, (n, rel)
    # the same step captured and replayed on other inputs
    zc, dc, mc = z.cuda(), dout.cuda(), m.cuda()
    step(layer, zc, mc, dev, dc, seed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z2, caught = step(layer, zc, mc, dev, dc, seed)
    for i in range(3):
        zc.copy_(synth.pair_tensor(N, dtype="bf16", seed=50 + i))
        graph.replay()
        torch.cuda.synchronize()
        caught_z2 = z2.clone()
        caught_dz = caught["z"].clone()
        eager, eager_grads = step(layer, zc, mc, dev, dc, seed)
        torch.cuda.synchronize()
        assert torch.equal(caught_z2, eager) and torch.equal(caught_dz, eager_grads["z"]), i
    layer.close()
