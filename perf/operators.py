"""What the rotary positions and the attention over packed sequences with shared key/value heads cost, as measured cases.

Every case is one pass through one operator, or through a run of them as a layer makes it:

  rotary   positions onto the query and key heads of a row (or, "inverse", the gradient back through them)
  forward  attention: output and row statistics
  backward attention: gradients of queries, keys and values from output, row statistics and the output's gradient
  layer    positions, attention, its gradient, the gradient back through the positions: a training step's share of one sub-block

Queries, keys and values lie side by side in the rows of one projection's output, as a layer leaves them; where the keys
are a stored context they are tensors of their own.  `own` False: plain torch operations in 32 bits.
"""
import math
import random

import torch

own = False

LOG2E = 1.4426950408889634

_ROT = dict(op="rotary", dtype="bf16", layout="half", base=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0,
            original=0, magnitude=1.0, first=0, period=0, given=False, inverse=False)
_ATT = dict(dtype="bf16", causal=True, ragged=False, lens=0)


def listed():
    return [
        # the next token of one sequence: a single row, far along
        dict(_ROT, name="rotary_one_token", rows=1, heads=32, kv=8, dh=128, dims=128, first=8191),
        # fp32, odd numbers of rows and heads, part of an odd head, neighbouring channels paired, positions given
        dict(_ROT, name="rotary_f32_odd", dtype="f32", rows=1000, heads=4, kv=1, dh=72, dims=36, layout="interleaved", given=True),
        # the small language model's batch: 128 sequences of 256, 4 heads of 64
        dict(_ROT, name="rotary_small_model", rows=128 * 256, heads=4, kv=4, dh=64, dims=64, period=256),
        # a long context stretched eightfold, half of every head rotated, the gradient's way back
        dict(_ROT, name="rotary_long_grad", rows=131072, heads=16, kv=8, dh=128, dims=64, base=500000.0, scaling="by_parts",
             factor=8.0, original=16384, magnitude=1.2, inverse=True),
        # reference precision: a handful of short documents packed together
        dict(_ATT, name="fwd_f32_packed", op="forward", dtype="f32", heads=4, kv=2, dh=32, seqs=9, lq=60, lk=60, ragged=True, lens=3),
        # documents of unequal length packed into one batch, four query heads to a key head
        dict(_ATT, name="fwd_packed", op="forward", heads=16, kv=4, dh=64, seqs=24, lq=700, lk=700, ragged=True, lens=5),
        # one new token for each of 32 sequences over their stored context
        dict(_ATT, name="fwd_tokens", op="forward", heads=32, kv=8, dh=128, seqs=32, lq=1, lk=4096),
        # one long document
        dict(_ATT, name="fwd_long", op="forward", heads=32, kv=8, dh=128, seqs=1, lq=16384, lk=16384),
        # the small language model's batch with one key head for all
        dict(_ATT, name="bwd_small_model", op="backward", heads=4, kv=1, dh=64, seqs=128, lq=256, lk=256),
        # the packed documents' gradient
        dict(_ATT, name="bwd_packed", op="backward", heads=16, kv=4, dh=64, seqs=24, lq=700, lk=700, ragged=True, lens=5),
        # a long document's gradient
        dict(_ATT, name="bwd_long", op="backward", heads=32, kv=8, dh=128, seqs=1, lq=8192, lk=8192),
        # a layer's share of a training step: 16 sequences of 1024, 16 heads of 64 on 4 key heads
        dict(_ROT, **dict(_ATT, name="layer_train", heads=16, kv=4, dh=64, dims=64, seqs=16, lq=1024, lk=1024, period=1024)) | dict(op="layer"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    fam = rng.choice(("rotary", "rotary", "forward", "tokens", "backward", "backward", "layer"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    dh = rng.choice((64, 64, 128, 128, 32, 80, 96, 8 * rng.randint(1, 16)))
    kv = rng.choice((1, 2, 4, 8, 3))
    group = rng.choice((1, 1, 2, 4, 4, 7, 8))
    heads = kv * group
    rot = {}
    if fam in ("rotary", "layer"):
        dims = dh if rng.random() < 0.5 else 2 * rng.randint(2, dh // 2)
        scaling = rng.choice(("none", "none", "linear", "base", "by_parts"))
        rot = dict(_ROT, dims=dims, layout=rng.choice(("half", "interleaved")), scaling=scaling, base=rng.choice((10000.0, 500000.0)),
                   factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)), original=4096 if scaling == "by_parts" else 0,
                   magnitude=1.0 if scaling != "by_parts" else 1.1)
    if fam == "rotary":
        rows = _log(rng, 1, max(2, min(200000, int(3.0e8 / (heads * dh)))))
        return dict(rot, dtype=dtype, rows=rows, heads=heads, kv=kv, dh=dh, given=rng.random() < 0.3, first=rng.randint(0, 5000),
                    period=rng.choice((0, 0, 128, 1000)), inverse=rng.random() < 0.5)
    if fam == "tokens":
        lk = _log(rng, 16, 32768)
        lq = rng.choice((1, 1, 1, 2, 5, 16))
        seqs = max(1, min(64, _log(rng, 1, 64), int(1.5e8 / (lk * kv * dh))))
        return dict(_ATT, op="forward", dtype=dtype, heads=heads, kv=kv, dh=dh, seqs=seqs, lq=lq, lk=lk, ragged=rng.random() < 0.5,
                    lens=rng.randint(0, 999))
    lq = _log(rng, 1, 8192)
    cap = (3.0e11 if dtype == "bf16" else 6.0e10) / (10.0 * heads * dh)         # pairs: the cost of a case stays bounded
    lq = max(1, min(lq, int(math.sqrt(cap))))
    seqs = max(1, min(_log(rng, 1, 64), int(cap / (lq * lq)), 32768 // lq + 1))
    att = dict(_ATT, dtype=dtype, causal=rng.random() < 0.7, heads=heads, kv=kv, dh=dh, seqs=seqs, lq=lq, lk=lq,
               ragged=rng.random() < 0.5, lens=rng.randint(0, 999))
    if fam == "layer":
        return dict(rot, **att) | dict(op="layer", dtype=dtype, period=lq)
    return dict(att, op=fam)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Queries and keys of every sequence.  Ragged: between 1 and twice the mean, and one sequence without any token; with as
    many keys as queries the two agree, otherwise a sequence has at least as many keys as queries."""
    n, lq, lk = case["seqs"], case["lq"], case["lk"]
    if not case["ragged"]:
        return [lq] * n, [lk] * n
    r = random.Random(case["lens"])
    if lq == lk:
        q = [r.randint(1, 2 * lq - 1) for _ in range(n)]
        if n >= 4:
            q[n // 2] = 0
        return q, list(q)
    return [lq] * n, [r.randint(lq, max(lq, 2 * lk - 1)) for _ in range(n)]


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(case)
    H, K, D = case["heads"], case["kv"], case["dh"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    if case["op"] == "rotary":
        s = dict(x=normal(case["rows"], H + 2 * K, D), positions=None)
        if case["given"]:
            s["positions"] = torch.randint(0, 100000, (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        return s
    lq, lk = _lengths(case)
    nq, nk = sum(lq), sum(lk)
    if case["lq"] == case["lk"]:
        qkv = normal(nq, H + 2 * K, D)
        s = dict(qkv=qkv, q=qkv[:, :H], k=qkv[:, H:H + K], v=qkv[:, H + K:])
    else:
        s = dict(q=normal(nq, H, D), k=normal(nk, K, D), v=normal(nk, K, D))
    s["lq"], s["lk"] = lq, lk
    if case["op"] != "forward":
        s["do"] = normal(nq, H, D)
    if case["op"] == "backward":
        s["o"], s["lse"] = _forward(s["q"], s["k"], s["v"], lq, lk, case["causal"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2501_17086_amd import binding as B
        H, K, D = case["heads"], case["kv"], case["dh"]
        if "dims" in case:
            s["rot"] = B.make_rotary(case["dims"], layout=case["layout"], base=case["base"], scaling=case["scaling"],
                                     factor=case["factor"], low=case["low"], high=case["high"], original=case["original"],
                                     magnitude=case["magnitude"])
        if case["op"] == "rotary":
            s["out"] = torch.empty((case["rows"], H + K, D), dtype=_type(case), device="cuda")
            return s
        q, k = s["q"], s["k"]
        if case["op"] == "layer":
            s["turned"] = torch.empty((q.shape[0], H + K, D), dtype=q.dtype, device="cuda")
            s["dturned"] = torch.empty_like(s["turned"])
            s["dqkv"] = torch.empty_like(s["qkv"])
            q, k = s["turned"][:, :H], s["turned"][:, H:]
        off = dict(q_offsets=_offsets(s["lq"]), k_offsets=_offsets(s["lk"])) if case["ragged"] else dict(seqs=case["seqs"])
        a = B.make_attention(q, k, s["v"], causal=case["causal"], o=s.get("o"), lse=s.get("lse"), grad=case["op"] != "forward", **off)
        if case["op"] == "layer":
            a.dq, a.dk, a.dv = s["dturned"][:, :H], s["dturned"][:, H:], s["dqkv"][:, H + K:]
        s["att"] = a
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    op, H, K = case["op"], case["heads"], case["kv"]
    if own:
        from paper_2501_17086_amd import binding as B
        if op == "rotary":
            B.hbp_rotary(s["rot"], s["x"][:, :H + K], s["out"], positions=s["positions"], first=case["first"], period=case["period"],
                         inverse=case["inverse"])
            return s["out"]
        a = s["att"]
        if op == "forward":
            B.hbp_attention_forward(a)
            return a.o, a.lse
        if op == "backward":
            B.hbp_attention_backward(a, s["do"])
            return a.dq, a.dk, a.dv
        B.hbp_rotary(s["rot"], s["qkv"][:, :H + K], s["turned"], first=case["first"], period=case["period"])
        B.hbp_attention_forward(a)
        B.hbp_attention_backward(a, s["do"])
        B.hbp_rotary(s["rot"], s["dturned"], s["dqkv"][:, :H + K], first=case["first"], period=case["period"], inverse=True)
        return a.o, s["dqkv"]
    if op == "rotary":
        return _rotary(case, s["x"][:, :H + K], s["positions"], case["inverse"])
    if op == "forward":
        return _forward(s["q"], s["k"], s["v"], s["lq"], s["lk"], case["causal"])
    if op == "backward":
        return _backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["lq"], s["lk"], case["causal"])
    turned = _rotary(case, s["qkv"][:, :H + K], None, False)
    q, k = turned[:, :H], turned[:, H:]
    o, lse = _forward(q, k, s["v"], s["lq"], s["lk"], case["causal"])
    dq, dk, dv = _backward(q, k, s["v"], o, lse, s["do"], s["lq"], s["lk"], case["causal"])
    dqk = _rotary(case, torch.cat((dq, dk), 1), None, True)
    return o, torch.cat((dqk, dv), 1)


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians per position of every channel pair, 64 bits."""
    n = case["dims"]
    i = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    base = case["base"]
    if case["scaling"] == "base":
        base = base * case["factor"] ** (n / (n - 2))
    f = torch.exp(i * (-2.0 / n) * math.log(base))
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "by_parts":
        w = ((case["original"] * f / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
        f = f * (w + (1 - w) / case["factor"])
    return f


def _positions(case, rows, given):
    if given is not None:
        return given.to(torch.float64)
    n = torch.arange(rows, device="cuda", dtype=torch.int64)
    if case["period"]:
        n = n % case["period"]
    return (n + case["first"]).to(torch.float64)


def _rotary(case, x, given, inverse):
    n = case["dims"]
    t = _positions(case, x.shape[0], given)[:, None] * _frequencies(case)
    c = (torch.cos(t) * case["magnitude"]).float()[:, None]
    s = (torch.sin(t) * (-case["magnitude"] if inverse else case["magnitude"])).float()[:, None]
    y = x.float()
    out = y.clone()
    if case["layout"] == "half":
        a, b = y[..., :n // 2], y[..., n // 2:n]
        out[..., :n // 2], out[..., n // 2:n] = a * c - b * s, a * s + b * c
    else:
        a, b = y[..., 0:n:2], y[..., 1:n:2]
        out[..., 0:n:2], out[..., 1:n:2] = a * c - b * s, a * s + b * c
    return out.to(x.dtype)


def _pieces(lq, lk, heads):
    """(sequence, its first query and key, first and last query of a piece): pieces whose scores take 1 GB at most."""
    q0 = k0 = 0
    for n, m in zip(lq, lk):
        step = max(1, min(n, (1 << 28) // max(1, heads * m)))
        for i in range(0, n, step):
            yield n, m, q0, k0, i, min(n, i + step)
        q0, k0 = q0 + n, k0 + m


def _unseen(n, m, i, j):
    """Where query i .. j of n does not see the m keys: the last query sees all of them."""
    qi = torch.arange(i, j, device="cuda")[:, None]
    return torch.arange(m, device="cuda")[None, :] > qi + (m - n)


def _heads_first(x, a, b):
    return x[a:b].float().transpose(0, 1).contiguous()


def _scores(q, k, n, m, q0, k0, i, j, causal):
    """Scaled scores of a piece, [key heads, group, queries, keys], -inf where not seen."""
    H, K, D = q.shape[1], k.shape[1], q.shape[2]
    qs = _heads_first(q, q0 + i, q0 + j).reshape(K, H // K * (j - i), D)
    ks = k[k0:k0 + m].float().permute(1, 2, 0).contiguous()
    s = torch.matmul(qs, ks).mul_(D ** -0.5).view(K, H // K, j - i, m)
    if causal:
        s.masked_fill_(_unseen(n, m, i, j), -math.inf)
    return s


def _forward(q, k, v, lq, lk, causal):
    N, H, D = q.shape
    K = k.shape[1]
    o = torch.zeros((N, H, D), dtype=q.dtype, device="cuda")
    lse = torch.full((N, H), -math.inf, device="cuda")
    for n, m, q0, k0, i, j in _pieces(lq, lk, H):
        if m == 0:
            continue
        s = _scores(q, k, n, m, q0, k0, i, j, causal)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        vs = _heads_first(v, k0, k0 + m)
        r = torch.matmul(p.view(K, -1, m), vs).view(K, H // K, j - i, D) / torch.where(total == 0, torch.ones_like(total), total)
        o[q0 + i:q0 + j] = r.reshape(H, j - i, D).transpose(0, 1).to(q.dtype)
        lse[q0 + i:q0 + j] = ((top + total.log()) * LOG2E).reshape(H, j - i).transpose(0, 1)
    return o, lse


def _backward(q, k, v, o, lse, do, lq, lk, causal):
    N, H, D = q.shape
    K = k.shape[1]
    dq = torch.zeros((N, H, D), dtype=q.dtype, device="cuda")
    dk = torch.zeros((k.shape[0], K, D), device="cuda")
    dv = torch.zeros((k.shape[0], K, D), device="cuda")
    scale = D ** -0.5
    for n, m, q0, k0, i, j in _pieces(lq, lk, H):
        if m == 0:
            continue
        p = _scores(q, k, n, m, q0, k0, i, j, causal)
        L = lse[q0 + i:q0 + j].transpose(0, 1).reshape(K, H // K, j - i, 1) / LOG2E
        p = p.sub_(torch.where(L == -math.inf, torch.zeros_like(L), L)).exp_()
        g = _heads_first(do, q0 + i, q0 + j)
        delta = (g * _heads_first(o, q0 + i, q0 + j)).sum(-1).view(K, H // K, j - i, 1)
        g = g.reshape(K, -1, D)
        ds = torch.matmul(g, v[k0:k0 + m].float().permute(1, 2, 0).contiguous()).view(p.shape).sub_(delta).mul_(p).view(K, -1, m)
        p = p.view(K, -1, m)
        dq[q0 + i:q0 + j] = torch.matmul(ds, _heads_first(k, k0, k0 + m)).mul_(scale).reshape(H, j - i, D).transpose(0, 1).to(q.dtype)
        qs = _heads_first(q, q0 + i, q0 + j).reshape(K, -1, D)
        dk[k0:k0 + m] += torch.matmul(ds.transpose(1, 2).contiguous(), qs).mul_(scale).transpose(0, 1)
        dv[k0:k0 + m] += torch.matmul(p.transpose(1, 2).contiguous(), g).transpose(0, 1)
    return dq, dk.to(q.dtype), dv.to(q.dtype)


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turn64(case, x, given, sign):
    """Every pair as a complex number times magnitude exp(+-i angle)."""
    n, rows = case["dims"], x.shape[0]
    pos = [case["first"] + (r % case["period"] if case["period"] else r) for r in range(rows)] if given is None else given.tolist()
    freq = []
    for i in range(n // 2):
        f = case["base"] ** (-2.0 * i / n)
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "base":
            f = (case["base"] * case["factor"] ** (n / (n - 2.0))) ** (-2.0 * i / n)
        elif case["scaling"] == "by_parts":
            turns = case["original"] * f / (2.0 * math.pi)
            w = min(1.0, max(0.0, (turns - case["low"]) / (case["high"] - case["low"])))
            f = w * f + (1.0 - w) * f / case["factor"]
        freq.append(f)
    angle = torch.outer(torch.tensor(pos, dtype=torch.float64), torch.tensor(freq, dtype=torch.float64)).cuda()
    factor = torch.polar(torch.full_like(angle, case["magnitude"]), sign * angle)[:, None, :]
    out = x.double().clone()
    lead = out[..., :n]
    pairs = lead.reshape(*lead.shape[:-1], 2, n // 2).transpose(-1, -2) if case["layout"] == "half" else \
        lead.reshape(*lead.shape[:-1], n // 2, 2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * factor)
    out[..., :n] = (turned.transpose(-1, -2) if case["layout"] == "half" else turned).reshape(lead.shape)
    return out


def _attend64(q, k, v, lq, lk, causal, do=None, o=None, lse=None):
    """Output and statistics; with do also the gradients, by the given o and lse where there are such.  Head by head."""
    N, H, D = q.shape
    group = H // k.shape[1]
    keep_o, keep_l = o, lse
    o = torch.zeros((N, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((N, H), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (q, k, v))
    a = b = 0
    for n, m in zip(lq, lk):
        for h in range(H if n and m else 0):
            kh, vh = k[b:b + m, h // group].double(), v[b:b + m, h // group].double()
            for i in range(0, n, 4096):
                j = min(n, i + 4096)
                row = slice(a + i, a + j)
                s = q[row, h].double() @ kh.T / math.sqrt(D)
                if causal:
                    limit = torch.arange(i, j, device="cuda") + (m - n)
                    s[torch.arange(m, device="cuda")[None, :] > limit[:, None]] = -math.inf
                l = torch.logsumexp(s, 1)
                lse[row, h] = l * LOG2E
                if keep_l is not None:
                    l = keep_l[row, h].double() / LOG2E
                p = torch.exp(s - torch.where(torch.isinf(l), torch.zeros_like(l), l)[:, None])
                oh = p @ vh
                o[row, h] = oh
                if do is not None:
                    g = do[row, h].double()
                    d = (g * (oh if keep_o is None else keep_o[row, h].double())).sum(1, keepdim=True)
                    ds = p * (g @ vh.T - d) / math.sqrt(D)
                    dq[row, h] = ds @ kh
                    dk[b:b + m, h // group] += ds.T @ q[row, h].double()
                    dv[b:b + m, h // group] += p.T @ g
        a, b = a + n, b + m
    return o, lse, dq, dk, dv


def exact(case, seed):
    s = _inputs(case, seed)
    op, H, K = case["op"], case["heads"], case["kv"]
    if op == "rotary":
        return _turn64(case, s["x"][:, :H + K], s["positions"], -1.0 if case["inverse"] else 1.0)
    if op == "forward":
        return _attend64(s["q"], s["k"], s["v"], s["lq"], s["lk"], case["causal"])[:2]
    if op == "backward":
        return _attend64(s["q"], s["k"], s["v"], s["lq"], s["lk"], case["causal"], s["do"], s["o"], s["lse"])[2:]
    turned = _turn64(case, s["qkv"][:, :H + K], None, 1.0)
    o, _, dq, dk, dv = _attend64(turned[:, :H], turned[:, H:], s["v"], s["lq"], s["lk"], case["causal"], s["do"])
    return o, torch.cat((_turn64(case, torch.cat((dq, dk), 1), None, -1.0), dv), 1)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    H, K, D = case["heads"], case["kv"], case["dh"]
    if case["op"] == "rotary":
        n = case["rows"] * (H + K)
        return {"bytes": 2.0 * n * D * es + (4.0 * case["rows"] if case["given"] else 0.0), "flops": 3.0 * n * case["dims"]}
    lq, lk = _lengths(case)
    nq, nk = sum(lq), sum(lk)
    if case["causal"]:
        pairs = sum(sum(max(0, min(m, i + 1 + m - n)) for i in range(n)) for n, m in zip(lq, lk))
    else:
        pairs = sum(n * m for n, m in zip(lq, lk))
    q, kv, stat = nq * H * D * es, nk * K * D * es, 4.0 * nq * H
    if case["op"] == "forward":
        return {"bytes": 2.0 * q + 2.0 * kv + stat, "flops": 4.0 * D * H * pairs}
    if case["op"] == "backward":
        return {"bytes": 4.0 * q + 4.0 * kv + stat, "flops": 10.0 * D * H * pairs}
    # q, k, v and do in; o and the three gradients out
    return {"bytes": 4.0 * q + 4.0 * kv, "flops": 14.0 * D * H * pairs + 6.0 * nq * (H + K) * case["dims"]}
