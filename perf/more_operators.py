"""What a training step does between the projections and the attention, and what it keeps, measured through public calls.

Three operators: the norm of queries and keys by head with the position
rotation (forward; forward and backward; the same with the inputs held in 8
bits in between), the relative position bias by buckets (as an attention bias
and added to a pair tensor; forward, and forward with the gradient of the table), and tensors
held in 8 bits with a power of two for each group.  listed() names twelve
calls, draw() takes more from the same ranges, exact() states the results in
float64.
"""
import math

import numpy as np
import torch

own = False      # True: the library's kernels; False: elementary torch operations

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # serving: one new token of each of 4 sequences far into their contexts, shared key heads: latency
        _norm("norm_rotate_fwd_tokens4", 4, 1, 16, 4, 64, 64, "bf16", "rms", "halves", "far"),
        # long sequences in front of the attention, wide heads
        _norm("norm_rotate_fwd_n6000_d128", 2, 6000, 16, 16, 128, 128, "bf16", "rms", "halves", "shared"),
        # a model run in float32 with odd lengths: narrow heads, two thirds of the channels turned, packed sequences
        _norm("norm_rotate_fwd_f32_n777_d24", 2, 777, 4, 2, 24, 16, "f32", "layer", "adjacent", "packed"),
        # training step of triangle attention on a usual crop: rows as batch, positions shared by them
        _norm("norm_rotate_train_triangle_n384", 384, 384, 4, 4, 32, 32, "bf16", "layer", "halves", "shared", op="train"),
        # training step of a long decoder with shared key heads, its q and k held in 8 bits until the backward
        _norm("norm_rotate_train8_n2048_gqa", 4, 2048, 16, 4, 128, 64, "bf16", "rms", "adjacent", "packed", op="train8"),
        # bias of a small crop: latency
        _bias("relative_bias_fwd_n64", 1, 64, 64, 4, "bf16", "clip", 32, 0, False, False),
        # decoder over another sequence's states: logarithmic buckets, added to a bias that is there
        _bias("relative_bias_fwd_q2048_k3000", 1, 2048, 3000, 16, "bf16", "log", 32, 128, False, True),
        # training: the bias, and its table's gradient from the attention's dbias; several chains, token counts as they come
        _bias("relative_bias_train_n1300", 1, 1300, 1300, 16, "bf16", "clip", 32, 0, True, False, train=True),
        # the pair tensor of a large complex of several chains
        _pair("relative_pair_fwd_n2048", 2048, 2048, 128, "bf16", "clip", 32, 0, True),
        # training: the same on one rectangular tile in float32, with the table's gradient
        _pair("relative_pair_train_f32_n500x700", 500, 700, 128, "f32", "clip", 32, 0, True, train=True),
        # the pair tensor that a layer keeps for its backward, written and read
        _checkpoint("checkpoint8_bf16_n1024", 1024 * 1024, 128, "bf16", 32),
        # small float32 tensor of odd width
        _checkpoint("checkpoint8_f32_n333_c30", 333, 30, "f32", 16),
    ]


def _norm(name, batch, n, heads, kv_heads, d, rot, dtype, norm, pairs, pos, op="norm"):
    return dict(name=name, op=op, batch=batch, n=n, heads=heads, kv_heads=kv_heads, d=d, rot=rot, dtype=dtype, norm=norm,
                pairs=pairs, pos=pos)


def _bias(name, batch, nq, nk, heads, dtype, kind, buckets, reach, chains, base, train=False):
    return dict(name=name, op="bias_train" if train else "bias", batch=batch, nq=nq, nk=nk, heads=heads, dtype=dtype, kind=kind,
                buckets=buckets, reach=reach, chains=chains, base=base)


def _pair(name, n, m, c, dtype, kind, buckets, reach, chains, train=False):
    return dict(name=name, op="pair_train" if train else "pair", batch=1, nq=n, nk=m, heads=c, dtype=dtype, kind=kind, buckets=buckets,
                reach=reach, chains=chains, base=True)


def _checkpoint(name, rows, n, dtype, group):
    return dict(name=name, op="checkpoint", rows=rows, n=n, dtype=dtype, group=group)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = 4 if dtype == "f32" else 2
    which = rng.random()
    if which < 0.4:
        op = rng.choice(["norm", "train", "train8"])
        heads = rng.choice([1, 2, 3, 4, 8, 16])
        kv_heads = heads if rng.random() < 0.6 else rng.choice([h for h in range(1, heads + 1) if heads % h == 0])
        d = rng.choice([8, 16, 24, 32, 40, 64, 64, 80, 96, 128, 256])
        rot = rng.choice([d, d, d // 16 * 8, 8])
        most = 8e7 / size / ((heads + kv_heads) * d)
        n = _log_int(rng, 1, min(8000, most))
        batch = _log_int(rng, 1, max(1, min(512, most / n)))
        case = _norm("", batch, n, heads, kv_heads, d, rot, dtype, rng.choice(["rms", "layer"]), rng.choice(["halves", "adjacent"]),
                     rng.choice(["shared", "packed", "far"]), op)
    elif which < 0.85:
        kind = rng.choice(["clip", "log", "log_past"])
        buckets, reach = (rng.randint(1, 64), 0) if kind == "clip" else (2 * rng.randint(4, 40), rng.choice([100, 128, 400, 1000]))
        chains = rng.random() < 0.5
        if rng.random() < 0.6:
            nq, nk = _log_int(rng, 1, 3000), _log_int(rng, 1, 3000)
            heads = rng.choice([1, 3, 4, 8, 12, 16])
            batch = 1 if chains else min(_log_int(rng, 1, 64), max(1, int(1e8 / (nq * nk * heads))))
            case = _bias("", batch, nq, nk, heads, dtype, kind, buckets, reach, chains, rng.random() < 0.5, train=rng.random() < 0.5)
        else:
            n, m, c = _log_int(rng, 8, 1000), _log_int(rng, 8, 1000), rng.choice([30, 64, 128, 128, 384])
            case = _pair("", n, m, c, dtype, kind, buckets, reach, chains, train=rng.random() < 0.5)
    else:
        n, group = rng.choice([8, 30, 64, 128, 128, 384, 1000]), rng.choice([16, 32, 32, 64, 128])
        case = _checkpoint("", _log_int(rng, 1, 1.5e8 / n), n, dtype, group)
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _generator(seed, sub):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + sub)
    return g


def _normal(shape, seed, sub, dtype):
    return torch.randn(shape, generator=_generator(seed, sub), device="cuda", dtype=torch.float32).to(dtype)


def _integers(shape, low, high, seed, sub):
    return torch.randint(low, high, shape, generator=_generator(seed, sub), device="cuda", dtype=torch.int32)


def _activations(shape, seed, sub, dtype):
    """What projections leave: channels of different scale, some of them far larger than the rest."""
    c = shape[-1]
    scale = torch.exp(0.5 * _normal((c,), seed, sub + 32, torch.float32))
    scale[:: max(c // 4, 1)] *= 6
    return (torch.randn(shape, generator=_generator(seed, sub), device="cuda", dtype=torch.float32) * scale).to(dtype)


def _chain_positions(n, seed, sub):
    """Chains one after the other, each counted from a start of its own with a gap here and there: positions, chain numbers."""
    rise = (torch.rand((n,), generator=_generator(seed, sub), device="cuda") < 0.01).to(torch.int32) * 5 + 1
    chain = (torch.arange(n, device="cuda") * 5 // max(n, 1)).to(torch.int32)
    pos = torch.cumsum(rise, 0).to(torch.int32)
    first = torch.searchsorted(chain, chain)
    return pos - pos[first] + 1, chain


def _lut(case):
    """The bucket of each distance key - query in [-D, D], and D.  clip: one for each distance.  log: half of the buckets for
    keys behind the query, of each half the first half for single distances, the rest spaced evenly in the logarithm up to
    `reach`; log_past: all buckets so for keys before the query, bucket 0 for those behind it."""
    if case["kind"] == "clip":
        return list(range(2 * case["buckets"] + 1)), case["buckets"]
    per = case["buckets"] // (2 if case["kind"] == "log" else 1)
    single, reach = per // 2, case["reach"]
    steps = per - single

    def bucket(r):
        if r < single:
            return r
        k = 0     # the largest k with (r / single)^steps >= (reach / single)^k, in whole numbers
        while k + 1 < steps and r ** steps >= reach ** (k + 1) * single ** (steps - k - 1):
            k += 1
        return single + k
    past = [bucket(r) for r in range(reach + 1)]
    ahead = [per + b for b in past] if case["kind"] == "log" else [0] * (reach + 1)
    return past[:0:-1] + [past[0]] + ahead[1:], reach


def _buckets(case):
    """Rows of the table: the buckets, and the one for pairs of two chains."""
    return (2 * case["buckets"] + 1 if case["kind"] == "clip" else case["buckets"]) + (1 if case["chains"] else 0)


def prepare(case, seed):
    op = case["op"]
    dt = _DT[case["dtype"]]
    if op == "checkpoint":
        return dict(case=case, x=_activations((case["rows"], case["n"]), seed, 1, dt))
    if op in ("norm", "train", "train8"):
        b, n, h, hk, d, rot = (case[t] for t in ("batch", "n", "heads", "kv_heads", "d", "rot"))
        qk = _activations((b, n, (h + hk) * d), seed, 1, dt)           # one projection gives both
        s = dict(case=case, q=qk[..., :h * d].unflatten(-1, (h, d)), k=qk[..., h * d:].unflatten(-1, (hk, d)),
                 freqs=torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda"))
        at = torch.arange(n, device="cuda", dtype=torch.int32)
        if case["pos"] == "shared":
            s["positions"] = at
        elif case["pos"] == "far":
            s["positions"] = (_integers((b, 1), 100000, 1000000, seed, 3) + at).contiguous()
        else:
            length = _integers((b, 1), 1, n + 1, seed, 3)
            s["positions"] = (at % length).contiguous()
        for i, x in enumerate("qk"):
            s["gain_" + x] = (1 + 0.2 * _normal((d,), seed, 4 + i, torch.float32)).to(dt)
            s["shift_" + x] = (0.2 * _normal((d,), seed, 6 + i, torch.float32)).to(dt) if case["norm"] == "layer" else None
        if op != "norm":
            s["dq"], s["dk"] = _normal((b, n, h, d), seed, 8, dt), _normal((b, n, hk, d), seed, 9, dt)
        return s
    b, nq, nk, h = (case[t] for t in ("batch", "nq", "nk", "heads"))
    lut, reach = _lut(case)
    s = dict(case=case, table=(0.5 * _normal((_buckets(case), h), seed, 1, torch.float32)).to(dt), seg_q=None, seg_k=None)
    if own:
        from paper_2603_14806_amd import relative
        if case["kind"] == "clip":
            s["plan"] = relative.Buckets.clipped(case["buckets"], other=case["chains"])
        else:
            s["plan"] = relative.Buckets.logarithmic(case["buckets"], reach, both=case["kind"] == "log", other=case["chains"])
    else:
        s["lut"], s["reach"] = torch.tensor(lut, device="cuda"), reach
    if case["chains"]:
        s["pos_k"], s["seg_k"] = _chain_positions(nk, seed, 2)
        s["pos_q"], s["seg_q"] = (s["pos_k"], s["seg_k"]) if nq == nk else _chain_positions(nq, seed, 3)
    else:
        s["pos_k"] = torch.arange(nk, device="cuda", dtype=torch.int32)
        s["pos_q"] = torch.arange(nq, device="cuda", dtype=torch.int32) + max(nk - nq, 0) // 2
        if b > 1:         # each entry is a window with a start of its own
            s["pos_q"] = (s["pos_q"] + _integers((b, 1), -200, 200, seed, 4)).contiguous()
    shape = (nq, nk, h) if op.startswith("pair") else (b, h, nq, -(-nk // 8) * 8)       # (the bias with padded rows)
    for i, (name, there) in enumerate((("base", case["base"]), ("dout", op.endswith("train")))):
        s[name] = _normal(shape, seed, 5 + i, dt) if there else None
        if there and op.startswith("bias"):
            s[name] = s[name][..., :nk]
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        return _run_own(case, state)
    dt = _DT[case["dtype"]]
    if op == "checkpoint":
        return _eight_bits(state["x"].float(), case["group"]).to(dt)
    if op in ("norm", "train", "train8"):
        return _norm_plain(case, state)
    bucket, pair = _bucket_plain(state), op.startswith("pair")
    out = state["table"].float()[bucket]
    out = out[0] if pair else out.permute(0, 3, 1, 2)
    out = (out if state["base"] is None else state["base"].float() + out).to(dt)
    if state["dout"] is None:
        return out
    rows, g = state["table"].shape[0], state["dout"]
    if pair:
        return dict(out=out, table=_sum_by_bucket(bucket.flatten(), g.flatten(0, 1), rows).float())
    each = [_sum_by_bucket(bucket[min(e, len(bucket) - 1)].flatten(), g[e].flatten(1).T, rows) for e in range(len(g))]
    return dict(out=out, table=torch.stack(each).sum(0).float())


def _run_own(case, s):
    op = case["op"]
    if op == "checkpoint":
        from paper_2603_14806_amd import checkpoint8
        return checkpoint8.pack(s["x"], case["group"]).unpack()
    if op in ("norm", "train", "train8"):
        from paper_2603_14806_amd import normrotate
        weights = dict(gain_q=s["gain_q"], gain_k=s["gain_k"], shift_q=s["shift_q"], shift_k=s["shift_k"])
        args = (s["positions"], s["freqs"])
        how = dict(norm=case["norm"], pairs=case["pairs"], eps=1e-6, **weights)
        if op == "train8":
            yq, yk, q, k = normrotate.norm_rotate(s["q"], s["k"], *args, checkpoint=True, **how)
        else:
            (yq, yk), q, k = normrotate.norm_rotate(s["q"], s["k"], *args, **how), s["q"], s["k"]
        if op == "norm":
            return dict(q=yq, k=yk)
        dq, dk, grads = normrotate.norm_rotate_backward(q, k, s["dq"], s["dk"], *args, **how)
        return dict(q=yq, k=yk, dq=dq, dk=dk, **grads)
    from paper_2603_14806_amd import relative
    where = (s["plan"], s["pos_q"], s["pos_k"], s["seg_q"], s["seg_k"])
    if op.startswith("pair"):
        forward, backward, how = relative.relative_pair, relative.relative_pair_backward, {}
    else:
        forward, backward, how = relative.relative_bias, relative.relative_bias_backward, dict(dtype=case["dtype"])
    out = forward(s["table"], *where, base=s["base"], **how)
    return out if s["dout"] is None else dict(out=out, table=backward(s["dout"], *where))


def _eight_bits(x, group):
    """The values that 8 bits and a power of two for each `group` of the last axis stand for."""
    n = x.shape[-1]
    full = torch.nn.functional.pad(x, (0, -n % group)).unflatten(-1, (-1, group))
    top, e = torch.frexp(full.abs().amax(-1, keepdim=True))           # top in [1/2, 1)
    k = torch.where(torch.round(top * 128) > 127, e - 6, e - 7).clamp(min=-127)
    low = k // 2                                                       # 2^k in two factors that float32 has
    code = torch.round(full * _power(-low) * _power(low - k))
    return (code * _power(low) * _power(k - low)).flatten(-2)[..., :n]


def _power(k):
    """2^k as float32 for whole numbers k in [-126, 127]."""
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)


def _turn(x, cos, sin, pairs):
    """The pairs of the first channels turned; x [b][n][h][d], cos and sin [b or 1][n][1][rot / 2]."""
    half = cos.shape[-1]
    y = x.clone()
    a, b = (slice(0, half), slice(half, 2 * half)) if pairs == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _norm_plain(case, s):
    pos = s["positions"] if s["positions"].dim() == 2 else s["positions"][None]
    angle = pos.double()[..., None, None] * s["freqs"]
    cos, sin = angle.cos().float(), angle.sin().float()
    layer = case["norm"] == "layer"
    result = {}
    for name in "qk":
        x, dt = s[name].float(), s[name].dtype
        gain, shift = s["gain_" + name].float(), s["shift_" + name]

        def normed(x):
            if layer:
                x = x - x.mean(-1, keepdim=True)
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
            return x * r, r
        u = normed(x)[0] * gain
        result[name] = _turn(u if shift is None else u + shift.float(), cos, sin, case["pairs"]).to(dt)
        if case["op"] == "norm":
            continue
        if case["op"] == "train8":
            x = _eight_bits(x, case["d"])
        u, r = normed(x)
        g = _turn(s["d" + name].float(), cos, -sin, case["pairs"])
        result["gain_" + name] = (g * u).sum((0, 1, 2), dtype=torch.float64).float()
        if layer:
            result["shift_" + name] = g.sum((0, 1, 2), dtype=torch.float64).float()
        else:
            result["shift_" + name] = None
        g = g * gain
        dx = g - u * (g * u).mean(-1, keepdim=True)
        if layer:
            dx = dx - g.mean(-1, keepdim=True)
        result["d" + name] = (dx * r).to(dt)
    return result


def _bucket_plain(s):
    """[b or 1][nq][nk] row numbers of the table."""
    q, k = (t.long() if t.dim() == 2 else t.long()[None] for t in (s["pos_q"], s["pos_k"]))
    b = s["lut"][(k[:, None, :] - q[:, :, None]).clamp(-s["reach"], s["reach"]) + s["reach"]]
    if s["seg_q"] is not None:
        b = torch.where(s["seg_q"][None, :, None] == s["seg_k"][None, None, :], b, s["table"].shape[0] - 1)
    return b


def _sum_by_bucket(bucket, values, rows):
    """[rows][c] sums (float64) of the values [p][c] of each bucket: products with zeros and ones, long sums in 64 bits."""
    total = torch.zeros((rows, values.shape[1]), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // rows)
    at = torch.arange(rows, device="cuda")
    for i in range(0, len(bucket), step):
        total += torch.mm((at[:, None] == bucket[i:i + step]).double(), values[i:i + step].double())
    return total


# ------------------------------------------------------------------ work

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "checkpoint":
        n = case["rows"] * case["n"]
        return {"bytes": n * 2 * e + 2 * (n + case["rows"] * -(-case["n"] // case["group"])), "flops": 4 * n}
    if op in ("norm", "train", "train8"):
        rows = case["batch"] * case["n"] * (case["heads"] + case["kv_heads"])
        n = rows * case["d"]
        moved = {"norm": 2 * e * n, "train": 5 * e * n, "train8": 4 * e * n + 2 * (n + rows)}[op]
        places = case["n"] * (1 if case["pos"] == "shared" else case["batch"]) * 4
        return {"bytes": moved + places, "flops": n * (10 if op == "norm" else 30)}
    n = case["batch"] * case["nq"] * case["nk"] * case["heads"]
    tensors = 1 + case["base"] + op.endswith("train")
    weights = _buckets(case) * case["heads"] * (e + 4 * op.endswith("train"))
    return {"bytes": n * e * tensors + weights, "flops": n * tensors}


# ------------------------------------------------------------------ float64

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "checkpoint":
        return _eight_bits_exact(s["x"].double(), case["group"])
    if op in ("norm", "train", "train8"):
        return _norm_exact(case, s)
    lut, reach = _lut(case)
    q, k = (s[t].cpu().numpy().astype(np.int64) for t in ("pos_q", "pos_k"))
    q, k = (t if t.ndim == 2 else t[None] for t in (q, k))
    table = s["table"].double()
    rows = table.shape[0]
    base, dout, pair = s["base"], s["dout"], op.startswith("pair")
    out, grad = [], torch.zeros_like(table)
    for e in range(case["batch"]):
        far = np.clip(np.subtract.outer(k[min(e, len(k) - 1)], q[min(e, len(q) - 1)]).T, -reach, reach)
        b = np.asarray(lut)[far + reach]
        if case["chains"]:
            b = np.where(np.equal.outer(s["seg_q"].cpu().numpy(), s["seg_k"].cpu().numpy()), b, rows - 1)
        b = torch.from_numpy(b).cuda()
        t = torch.nn.functional.embedding(b, table) if pair else torch.stack([table[:, h][b] for h in range(case["heads"])])
        out.append(t if base is None else (base if pair else base[e]).double() + t)
        for r in range(rows if dout is not None else 0):
            grad[r] += dout[b == r].double().sum(0) if pair else dout[e][:, b == r].double().sum(1)
    out = out[0] if pair else torch.stack(out)
    return out if dout is None else dict(out=out, table=grad)


def _eight_bits_exact(x, group):
    out = torch.empty_like(x)
    for i in range(0, x.shape[-1], group):
        part = x[..., i:i + group]
        top = part.abs().amax(-1, keepdim=True)
        k = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 6
        for _ in range(2):         # (a logarithm next to a power of two may have fallen on its other side)
            k = torch.where(torch.round(top * torch.exp2(-k)) > 127, k + 1, k)
        k = torch.where(torch.round(top * torch.exp2(1 - k)) <= 127, k - 1, k)
        k = torch.where(top > 0, k, -127.0).clamp(min=-127)
        out[..., i:i + group] = torch.round(part * torch.exp2(-k)) * torch.exp2(k)
    return out


def _norm_exact(case, s):
    pos = s["positions"] if s["positions"].dim() == 2 else s["positions"][None]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[..., None] * s["freqs"])[:, :, None]
    rot, d = case["rot"], case["d"]

    def forward(x, gain, shift):
        if case["norm"] == "layer":
            u = torch.nn.functional.layer_norm(x, (d,), gain, shift, 1e-6)
        else:
            u = gain * x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + 1e-6)
        w = u[..., :rot]
        w = w.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["pairs"] == "halves" else w.unflatten(-1, (rot // 2, 2))
        w = torch.view_as_real(torch.complex(w[..., 0], w[..., 1]) * turn)
        w = w.transpose(-1, -2).flatten(-2) if case["pairs"] == "halves" else w.flatten(-2)
        return torch.cat([w, u[..., rot:]], -1)
    result = {}
    for name in "qk":
        x, gain = s[name].double(), s["gain_" + name].double()
        shift = None if s["shift_" + name] is None else s["shift_" + name].double()
        result[name] = forward(x, gain, shift)
        if case["op"] == "norm":
            continue
        if case["op"] == "train8":
            x = _eight_bits_exact(x, d)
        leaves = [t.clone().requires_grad_() for t in ([x, gain] if shift is None else [x, gain, shift])]
        grads = torch.autograd.grad(forward(*leaves, *[None] * (3 - len(leaves))), leaves, s["d" + name].double())
        result["d" + name], result["gain_" + name] = grads[:2]
        result["shift_" + name] = grads[2] if len(grads) > 2 else None
    return result
