"""What the two ends of a language model cost: embedding, dropout, and the cross entropy over its vocabulary, as measured cases.

Every case is one pass through one operator, or through a run of them as a training step makes it:

  dropout     elements left out by a counter-based generator, the rest scaled, added to a residual stream (or not)
  embed       rows of a table looked up by token, scaled, dropout on the way
  embed_grad  the table's gradient in 32 bits: rows of the same token added up, every other row of the table cleared
  loss        cross entropy of rows against a vocabulary: mean and every row's
  loss_grad   the same, with the gradients of the rows and of the vocabulary's weights, in the weights' type
  ends        a model whose table serves both ends: embedding with dropout, loss and its gradients, and the embedding's gradient on
              top of the vocabulary's

Tokens are drawn as text has them: the v-th most frequent one about 1 / v as often as the first.  A token or target of -1 is padding.
`own` False: plain torch operations in 32 bits.
"""
import math
import random

import numpy as np
import torch

own = False

_DROP = dict(op="dropout", dtype="bf16", rate=0.1, residual=False, strided=False)
_EMB = dict(dtype="bf16", rate=0.0, scaled=False, padding=0.0)
_LOSS = dict(dtype="bf16", padding=0.0, mean=True)


def listed():
    return [
        # one short sequence of the small language model
        dict(_DROP, name="dropout_small", rows=256, width=256),
        # fp32, odd sizes, part of a wider row, half of the elements left out
        dict(_DROP, name="dropout_f32_odd", dtype="f32", rows=1001, width=72, rate=0.5, strided=True),
        # a block's output on its way into a wide residual stream
        dict(_DROP, name="dropout_wide", rows=16384, width=2048, residual=True),
        # the next token of 32 sequences
        dict(_EMB, name="embed_tokens", op="embed", rows=32, vocab=16384, width=1024),
        # the small language model's batch: 128 sequences of 256, a vocabulary of 16384, with dropout
        dict(_EMB, name="embed_small_model", op="embed", rows=128 * 256, vocab=16384, width=256, rate=0.1, scaled=True),
        # its gradient
        dict(_EMB, name="embed_grad_small_model", op="embed_grad", rows=128 * 256, vocab=16384, width=256, rate=0.1, scaled=True),
        # a batch of a wide model over a large vocabulary, a tenth of it padding
        dict(_EMB, name="embed_grad_wide", op="embed_grad", rows=16384, vocab=131072, width=2048, padding=0.1),
        # scoring a handful of tokens
        dict(_LOSS, name="loss_tokens", op="loss", rows=8, vocab=16384, width=256),
        # reference precision, sizes that are no multiple of anything, padding
        dict(_LOSS, name="loss_grad_f32_odd", op="loss_grad", dtype="f32", rows=333, vocab=1009, width=72, padding=0.1),
        # a medium model on packed text, an odd vocabulary
        dict(_LOSS, name="loss_grad_odd", op="loss_grad", rows=8190, vocab=50021, width=1024, padding=0.05),
        # a wide model's batch over a large vocabulary
        dict(_LOSS, name="loss_grad_wide", op="loss_grad", rows=16384, vocab=131072, width=2048),
        # the small language model's training step outside its blocks, one table for both ends
        dict(_EMB, name="ends_small_model", op="ends", rows=128 * 256, vocab=16384, width=256, rate=0.1, scaled=True, mean=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("dropout", "embed", "embed_grad", "embed_grad", "loss", "loss_grad", "loss_grad", "ends"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    width = 8 * _log(rng, 2, 256)
    if rng.random() < 0.5:
        width = rng.choice((64, 128, 256, 512, 768, 1024, 2048))
    rate = rng.choice((0.0, 0.1, 0.1, 0.3, 0.5))
    if op == "dropout":
        return dict(_DROP, dtype=dtype, rows=_log(rng, 1, min(65536, (1 << 25) // width)), width=width, rate=rate or 0.2,
                    residual=rng.random() < 0.5, strided=rng.random() < 0.3)
    vocab = _log(rng, 50, 131072)
    if rng.random() < 0.3:
        vocab = rng.choice((256, 16384, 32768, 65536))
    padding = rng.choice((0.0, 0.0, 0.1, 0.5))
    if op in ("embed", "embed_grad"):
        return dict(_EMB, op=op, dtype=dtype, rows=_log(rng, 1, min(65536, (1 << 25) // width)), vocab=vocab, width=width, rate=rate,
                    scaled=rng.random() < 0.5, padding=padding)
    cap = (1.0e12 if dtype == "bf16" else 3.0e10) / width / vocab                 # products: the cost of a case stays bounded
    rows = max(1, min(int(cap), _log(rng, 1, 32768)))
    if op == "ends":
        return dict(_EMB, op=op, dtype=dtype, rows=rows, vocab=vocab, width=width, rate=rate, scaled=True, padding=padding, mean=True)
    return dict(_LOSS, op=op, dtype=dtype, rows=rows, vocab=vocab, width=width, padding=padding, mean=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _scale(case):
    return math.sqrt(case["width"]) if case["scaled"] else 1.0


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(case)
    op, N, D = case["op"], case["rows"], case["width"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)

    def tokens():
        u = torch.rand(N, generator=gen, device="cuda", dtype=torch.float64)
        t = (u * math.log(case["vocab"] + 1)).exp().floor().long().clamp_(1, case["vocab"]) - 1
        if case["padding"]:
            t[torch.rand(N, generator=gen, device="cuda") < case["padding"]] = -1
        return t.to(torch.int32)

    s = dict(seed=seed * 0x9E3779B97F4A7C15 % (1 << 64))
    if op == "dropout":
        s["x"] = normal(N, 2 * D)[:, :D] if case["strided"] else normal(N, D)
        if case["residual"]:
            s["residual"] = normal(N, D)
        return s
    s["tokens"] = tokens()
    if op == "embed_grad":
        s["table"] = torch.empty((case["vocab"], D), dtype=dt, device="cuda")
        s["dout"] = normal(N, D)
        return s
    s["table"] = normal(case["vocab"], D, std=0.02)
    if op in ("loss", "loss_grad"):
        # states that have learnt something: the target's logit stands out by 0 .. 12
        known = torch.rand(N, generator=gen, device="cuda") * (12.0 / (0.02 * 0.02 * D))
        s["x"] = (torch.randn((N, D), generator=gen, device="cuda") +
                  known[:, None] * s["table"][s["tokens"].long().clamp_(min=0)].float()).to(dt)
    if op == "ends":
        s["targets"] = tokens()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2501_17086_amd import binding as B
        op, rate = case["op"], case.get("rate", 0.0)
        drop = B.make_dropout(rate, seed=s["seed"], offset=3) if rate else None
        if op == "dropout":
            s["dropout"] = drop
            s["out"] = torch.empty((case["rows"], case["width"]), dtype=_type(case), device="cuda")
        if op in ("embed", "embed_grad", "ends"):
            s["embedding"] = B.make_embedding(s["tokens"], s["table"], scale=_scale(case), dropout=drop, grad=op != "embed",
                                              dtable=torch.empty_like(s["table"]) if op == "ends" else None)
        if op in ("loss", "loss_grad"):
            s["loss"] = B.make_cross_entropy(s["x"], s["table"], s["tokens"], mean=case["mean"], grad=op == "loss_grad",
                                             dweight=torch.empty_like(s["table"]) if op == "loss_grad" else None)
        if op == "ends":
            e = s["embedding"]
            s["loss"] = B.make_cross_entropy(e.out, s["table"], s["targets"], mean=case["mean"], dweight=e.dtable)
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2501_17086_amd import binding as B
        if op == "dropout":
            B.hbp_dropout(s["dropout"], s["x"], s["out"], residual=s.get("residual"))
            return s["out"]
        if op == "embed":
            B.hbp_embedding_forward(s["embedding"])
            return s["embedding"].out
        if op == "embed_grad":
            B.hbp_embedding_backward(s["embedding"], s["dout"])
            return s["embedding"].dtable
        c = s["loss"]
        if op == "ends":
            e = s["embedding"]
            B.hbp_embedding_forward(e)
            B.hbp_loss_cross_entropy(c)
            B.hbp_embedding_backward(e, c.dx, accumulate=True)
            return c.loss, c.row_loss, e.out, c.dx, e.dtable
        B.hbp_loss_cross_entropy(c)
        return (c.loss, c.row_loss) if op == "loss" else (c.loss, c.row_loss, c.dx, c.dweight)
    if op == "dropout":
        return _dropout(s["x"], case["rate"], s["seed"], s.get("residual"))
    if op == "embed":
        return _embed(case, s)
    if op == "embed_grad":
        return _embed_grad(case, s, s["dout"])
    if op in ("loss", "loss_grad"):
        return _loss(s["x"], s["table"], s["tokens"], case["mean"], op == "loss_grad")
    out = _embed(case, s)
    loss, rows, dx, dw = _loss(out, s["table"], s["targets"], case["mean"], True)
    return loss, rows, out, dx, (dw.float() + _embed_grad(case, s, dx)).to(dw.dtype)


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
_LOW = 0xFFFFFFFF


def _kept(rows, width, rate, seed, offset=3):
    """1 where an element stays, 0 where it is left out, [rows, width]: the counter-based generator Philox4x32-10, eight elements of a
    row to a call, 16 bits each (products of 32-bit words wrap in 64 bits, which the masks undo)."""
    block = torch.arange(rows * width // 8, device="cuda", dtype=torch.int64)
    c = [block & _LOW, block >> 32, torch.full_like(block, offset & _LOW), torch.full_like(block, offset >> 32)]
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) & _LOW ^ c[1] ^ k0, q & _LOW, (p >> 32) & _LOW ^ c[3] ^ k1, p & _LOW]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    w = torch.stack(c, 1)
    halves = torch.stack((w & 0xFFFF, w >> 16), 2)
    return (halves >= _threshold(rate)).view(rows, width)


def _threshold(rate):
    return int(round(rate * 65536))


def _dropout(x, rate, seed, residual=None):
    y = x.float() * _kept(*x.shape, rate, seed) * (65536.0 / (65536 - _threshold(rate)))
    if residual is not None:
        y = y + residual.float()
    return y.to(x.dtype)


def _coefficients(case, s):
    """What a token's row of the table is multiplied by, element by element."""
    c = (s["tokens"] >= 0).float()[:, None] * _scale(case)
    if case["rate"]:
        c = c * _kept(case["rows"], case["width"], case["rate"], s["seed"]) * (65536.0 / (65536 - _threshold(case["rate"])))
    return c


def _embed(case, s):
    return (s["table"][s["tokens"].long().clamp(min=0)].float() * _coefficients(case, s)).to(s["table"].dtype)


def _embed_grad(case, s, dout):
    g = torch.zeros((case["vocab"], case["width"]), device="cuda")
    return g.index_add_(0, s["tokens"].long().clamp(min=0), dout.float() * _coefficients(case, s))


def _loss(x, weight, targets, mean, grad):
    """In pieces of the vocabulary whose logits take 1 GB at most: running maximum and sum; then each piece once more for the gradients."""
    N, V = x.shape[0], weight.shape[0]
    step = max(1, min(V, (1 << 28) // N))
    xf, t = x.float(), targets.long()
    counts = t >= 0
    top = torch.full((N,), -math.inf, device="cuda")
    total = torch.zeros(N, device="cuda")
    for v in range(0, V, step):
        s = xf @ weight[v:v + step].float().t()
        new = torch.maximum(top, s.amax(1))
        total = total * (top - new).exp() + s.sub_(new[:, None]).exp_().sum(1)
        top = new
    lse = top + total.log()
    rows = torch.where(counts, lse - (xf * weight[t.clamp(min=0)].float()).sum(1), torch.zeros_like(lse))
    factor = 1.0 / counts.sum().clamp(min=1).float() if mean else torch.ones((), device="cuda")
    loss = (rows.double().sum().float() * factor).view(1)
    if not grad:
        return loss, rows
    dx = torch.zeros_like(xf)
    dw = torch.empty(weight.shape, device="cuda")
    each = (counts.float() * factor)[:, None]
    for v in range(0, V, step):
        w = weight[v:v + step].float()
        p = (xf @ w.t()).sub_(lse[:, None]).exp_()
        here = ((t >= v) & (t < v + w.shape[0])).nonzero()[:, 0]
        p[here, t[here] - v] -= 1.0
        p *= each
        dx += p @ w
        dw[v:v + step] = p.t() @ xf
    return loss, rows, dx.to(x.dtype), dw.to(weight.dtype)


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _multipliers64(rows, width, rate, seed, offset=3):
    """0 where an element is left out, else 1 / (share that stays): the generator once more, on the host in unsigned words."""
    limit = int(rate * 65536 + 0.5)
    n = rows * width // 8
    u32, u64 = np.uint32, np.uint64
    state = np.empty((4, n), dtype=u32)
    index = np.arange(n, dtype=u64)
    state[0], state[1] = index.astype(u32), (index >> u64(32)).astype(u32)
    state[2], state[3] = offset % 2 ** 32, offset // 2 ** 32
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        a = state[0].astype(u64) * u64(0xD2511F53)
        b = state[2].astype(u64) * u64(0xCD9E8D57)
        state = np.stack(((b >> u64(32)).astype(u32) ^ state[1] ^ u32(key[0]), b.astype(u32),
                          (a >> u64(32)).astype(u32) ^ state[3] ^ u32(key[1]), a.astype(u32)))
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.ascontiguousarray(state.T).view("<u2").reshape(rows, width)
    return torch.from_numpy(bits >= limit).cuda().double() * (65536.0 / (65536 - limit))


def _embed64(case, s):
    out = s["table"].double()[s["tokens"].clamp(min=0).long()] * _scale(case)
    if case["rate"]:
        out *= _multipliers64(case["rows"], case["width"], case["rate"], s["seed"])
    out[s["tokens"] < 0] = 0.0
    return out


def _embed_grad64(case, s, dout):
    """Tokens in order, running sums, and their differences between the ends of each token's stretch."""
    d = dout.double() * _scale(case)
    if case["rate"]:
        d *= _multipliers64(case["rows"], case["width"], case["rate"], s["seed"])
    order = torch.argsort(s["tokens"], stable=True)
    edges = torch.searchsorted(s["tokens"][order].contiguous(), torch.arange(case["vocab"] + 1, dtype=torch.int32, device="cuda"))
    out = torch.empty((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
    for c in range(0, case["width"], 256):
        sums = torch.cumsum(d[order, c:c + 256], 0)
        sums = torch.cat((torch.zeros_like(sums[:1]), sums))
        out[:, c:c + 256] = sums[edges[1:]] - sums[edges[:-1]]
    return out


def _loss64(x, weight, targets, mean, grad):
    """Some rows at a time against the whole vocabulary."""
    N, V = x.shape[0], weight.shape[0]
    w = weight.double()
    counted = int((targets >= 0).sum())
    each = 1.0 / max(1, counted) if mean else 1.0
    rows = torch.zeros(N, dtype=torch.float64, device="cuda")
    dx = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros(weight.shape, dtype=torch.float64, device="cuda") if grad else None
    step = max(1, (1 << 27) // V)
    for i in range(0, N, step):
        some = torch.arange(i, min(N, i + step), device="cuda")
        some = some[targets[some] >= 0]
        if some.numel() == 0:
            continue
        xs, ts = x[some].double(), targets[some].long()[:, None]
        logp = torch.log_softmax(xs @ w.T, 1)
        rows[some] = -logp.gather(1, ts)[:, 0]
        if grad:
            g = logp.exp_().scatter_add_(1, ts, torch.full(ts.shape, -1.0, dtype=torch.float64, device="cuda")) * each
            dx[some] = g @ w
            dw += g.T @ xs
    loss = (rows.sum() * each).view(1)
    return (loss, rows, dx, dw) if grad else (loss, rows)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "dropout":
        y = s["x"].double() * _multipliers64(case["rows"], case["width"], case["rate"], s["seed"])
        return y + s["residual"].double() if case["residual"] else y
    if op == "embed":
        return _embed64(case, s)
    if op == "embed_grad":
        return _embed_grad64(case, s, s["dout"])
    if op in ("loss", "loss_grad"):
        return _loss64(s["x"], s["table"], s["tokens"], case["mean"], op == "loss_grad")
    # (an operator reads what the one before it returned, in the storage type)
    out = _embed64(case, s)
    loss, rows, dx, dw = _loss64(out.to(_type(case)), s["table"], s["targets"], case["mean"], True)
    return loss, rows, out, dx, dw + _embed_grad64(case, s, dx.to(_type(case)))


def _distinct(case):
    """How many rows of the table a batch looks up, on the average."""
    v = np.arange(case["vocab"], dtype=np.float64)
    p = np.log((v + 2) / (v + 1)) / math.log(case["vocab"] + 1) * (1 - case["padding"])
    return float(-np.expm1(case["rows"] * np.log1p(-p)).sum())


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    op, N, D = case["op"], case["rows"], case["width"]
    rows = N * D * es
    if op == "dropout":
        return {"bytes": rows * (3.0 if case["residual"] else 2.0), "flops": N * D * (2.0 if case["residual"] else 1.0)}
    V = case["vocab"]
    if op == "embed":
        return {"bytes": 4.0 * N + _distinct(case) * D * es + rows, "flops": 1.0 * N * D}
    if op == "embed_grad":                                  # padding's rows are not read
        return {"bytes": 4.0 * N + rows * (1 - case["padding"]) + 4.0 * V * D, "flops": 1.0 * N * D}
    counted = N * (1 - case["padding"])
    if op == "loss":
        return {"bytes": 8.0 * N + rows + V * D * es, "flops": 2.0 * counted * V * D}
    if op == "loss_grad":                                   # logits, and the two gradients' products
        return {"bytes": 8.0 * N + 2.0 * rows + 2.0 * V * D * es, "flops": 6.0 * counted * V * D}
    return {"bytes": 12.0 * N + 2.0 * rows + 2.0 * V * D * es, "flops": 6.0 * counted * V * D + 2.0 * N * D}
