"""fp64 CPU oracle for attention of queries over keys of another length
(Fold-CP, Section 3.6, Eq. 6, with the queries and the keys two sequences).

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import or call
this module.  It shares no code, constants or helpers with the HIP library.

For batch entry b, query i, head h and key head g = h // (H / Hk):

    x_ij   = scale q_bih . k_bjg + bias_bhij        over keys j with m_bj = 1
    out_bih = sum_j softmax_j(x_ij) v_bjg           (no key left: 0)

and for a gradient `dout` of out, with P the softmax weights and
D_i = dout_bih . out_bih:

    dS_ij = P_ij (dout_bih . v_bjg - D_i)
    dq = scale sum_j dS_ij k_j, dk = scale sum_i dS_ij q_i, dv = sum_i P_ij dout_i

dk and dv are sums over the query heads of a key head, the gradient of a bias
the sum of dS over the axes the bias is shared along (length 1 in its shape).
Layouts: q, out [B][nq][H][d], k, v [B][nk][Hk][d], bias [B|1][H|1][nq][nk],
mask [B|1][nk].  Absent keys take no part whatever their k, v and bias hold.
"""
import numpy as np

from .trimul import f64


def _prepare(q, k, v, bias, mask, scale, rounded):
    q, k, v = f64(q), f64(k), f64(v)
    B, nq, H, d = q.shape
    nk, Hk = k.shape[1], k.shape[2]
    m = np.ones((B, nk), dtype=bool) if mask is None else np.broadcast_to(np.asarray(mask) != 0, (B, nk))
    k = np.where(m[:, :, None, None], k, 0.0)
    v = np.where(m[:, :, None, None], v, 0.0)
    kh = np.repeat(k.transpose(0, 2, 1, 3), H // Hk, axis=1)            # [B][H][nk][d]
    vh = np.repeat(v.transpose(0, 2, 1, 3), H // Hk, axis=1)
    qh = q.transpose(0, 2, 1, 3)
    x = np.matmul(qh, kh.transpose(0, 1, 3, 2)) * (d ** -0.5 if scale is None else scale)
    if bias is not None:
        x = x + np.where(m[:, None, None, :], f64(bias), 0.0)
    if rounded:      # the scores as float32 holds them: a huge bias swallows q . k
        x = x.astype(np.float32).astype(np.float64)
    x = np.where(m[:, None, None, :], x, -np.inf)
    return qh, kh, vh, x


def softmax_weights(x):
    """Softmax along the last axis; a row of -inf alone gives 0."""
    if x.shape[-1] == 0:
        return x
    top = x.max(axis=-1, keepdims=True)
    p = np.exp(x - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(axis=-1, keepdims=True)
    return np.divide(p, total, out=np.zeros_like(p), where=total > 0)


def cross_attention(q, k, v, bias=None, mask=None, scale=None, rounded=False):
    """out [B][nq][H][d] (float64)."""
    _, _, vh, x = _prepare(q, k, v, bias, mask, scale, rounded)
    return np.matmul(softmax_weights(x), vh).transpose(0, 2, 1, 3)


def cross_attention_backward(q, k, v, dout, bias=None, mask=None, scale=None, rounded=False):
    """dict of dq, dk, dv, dbias (None without a bias), and of what the gradients are made of: the weights P,
    dS, [B][H][nq][nk]."""
    qh, kh, vh, x = _prepare(q, k, v, bias, mask, scale, rounded)
    B, H, nq, d = qh.shape
    nk, Hk = np.shape(k)[1], np.shape(k)[2]
    s = d ** -0.5 if scale is None else scale
    P = softmax_weights(x)
    g = f64(dout).transpose(0, 2, 1, 3)
    D = (g * np.matmul(P, vh)).sum(-1, keepdims=True)
    dS = P * (np.matmul(g, vh.transpose(0, 1, 3, 2)) - D)
    dq = np.matmul(dS, kh).transpose(0, 2, 1, 3) * s
    dk = np.matmul(dS.transpose(0, 1, 3, 2), qh) * s
    dv = np.matmul(P.transpose(0, 1, 3, 2), g)
    dk, dv = (t.reshape(B, Hk, H // Hk, nk, d).sum(2).transpose(0, 2, 1, 3) for t in (dk, dv))
    dbias = None
    if bias is not None:
        dbias = dS
        for axis in (0, 1):
            if np.shape(bias)[axis] == 1:
                dbias = dbias.sum(axis, keepdims=True)
    return dict(dq=dq, dk=dk, dv=dv, dbias=dbias, P=P, dS=dS)
