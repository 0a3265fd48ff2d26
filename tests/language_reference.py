"""Embedding, dropout and cross entropy in 64 bits from the definitions, with bounds on what the library's roundings can come to.
Runs on the CPU or the GPU.

Roundings counted (u = half a step of the storage type, bf16 2^-8; f = 2^-24, half a step of fp32):
  product  f of itself, and f for a factor that was itself rounded to fp32
  sums     (number of terms + 4) f of the sum of the absolute terms, whatever their order
  logit    (width + 3) f of sum |x w| scale
  row sum  the logits' errors, (vocab + 16) f of the sum (its terms, each exponential 4 f, its exponent rounded), and 4 f of the
           logarithm's size; exponents go through base 2, one rounding of a logit's size
  dS       the errors of logit and row sum times the probability, 8 f; bf16: rounded once more, u
  result   u of itself
"""
import math

import numpy as np
import torch

F = 2.0 ** -24
TINY = 1e-38


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def assert_within(got, want, bound, what):
    got = got.double()
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {i}: {got[i].item()} for {want[i].item()}, "
                             f"off {off[i].item():.3g}, bound {bound[i].item():.3g}")


def philox(key, counter):
    """Four 32-bit words of Philox4x32-10 in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(rate) -> int:
    return round(float(np.float32(rate)) * 65536)


def kept(rows, width, rate, seed, offset=0):
    """True where an element stays, [rows, width] on the CPU, in numpy's unsigned words."""
    n = rows * width // 8
    block = np.arange(n, dtype=np.uint64)
    c = [block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), np.full(n, offset & 0xFFFFFFFF, np.uint64),
         np.full(n, offset >> 32, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack(c, 1)
    bits = np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), 2).reshape(rows, width)
    return torch.from_numpy(bits >= threshold(rate))


def multipliers(rows, width, drop, device):
    """What dropout multiplies by, 64 bits; drop: (rate, seed, offset) or None."""
    if drop is None or drop[0] == 0:
        return torch.ones((rows, width), dtype=torch.float64, device=device)
    rate, seed, offset = drop
    return kept(rows, width, rate, seed, offset).to(device).double() * (65536.0 / (65536 - threshold(rate)))


def dropout(x, drop, residual=None):
    """(output, bound)."""
    m = multipliers(*x.shape, drop, x.device)
    y = torch.where(m > 0, x.double() * m, torch.zeros_like(m))
    size = y.abs()
    if residual is not None:
        y = y + residual.double()
        size = size + residual.double().abs()
    return y, half_step(x.dtype) * y.abs() + 3 * F * size + TINY


def embedding(tokens, table, scale, drop=None):
    ok = (tokens >= 0) & (tokens < table.shape[0])
    rows = table.double()[torch.where(ok, tokens, torch.zeros_like(tokens)).long()]
    m = multipliers(tokens.numel(), table.shape[1], drop, table.device)
    y = torch.where(ok[:, None] & (m > 0), rows * m * scale, torch.zeros_like(m))
    return y, (half_step(table.dtype) + 3 * F) * y.abs() + TINY


def embedding_grad(tokens, dout, vocab, scale, drop, dtype, old=None):
    """dtable in `dtype`, added to `old` if there is one."""
    ok = (tokens >= 0) & (tokens < vocab)
    m = multipliers(*dout.shape, drop, dout.device)
    d = torch.where(m > 0, dout.double() * m * scale, torch.zeros_like(m))[ok]
    t = tokens[ok].long()
    want = torch.zeros((vocab, dout.shape[1]), dtype=torch.float64, device=dout.device)
    size, count = torch.zeros_like(want), torch.zeros(vocab, dtype=torch.float64, device=dout.device)
    want.index_add_(0, t, d)
    size.index_add_(0, t, d.abs())
    count.index_add_(0, t, torch.ones(t.shape, dtype=torch.float64, device=dout.device))
    bound = (count[:, None] + 6) * F * size
    if old is not None:
        want = want + old.double()
        bound = bound + 2 * F * (size + old.double().abs())
        bound[count == 0] = 0                               # rows without tokens stay as they are
        rounding = half_step(dtype) * want.abs() * (count > 0).double()[:, None]
    else:
        rounding = half_step(dtype) * want.abs()
    return want, bound + (rounding if dtype != torch.float32 else 0) + TINY * (count > 0).double()[:, None]


def cross_entropy(x, weight, targets, scale=1.0, mean=True, factor=1.0, grad_dtype=torch.float32):
    """{name: (value, bound)} of loss, row_loss, dx, dweight."""
    N, D = x.shape
    V = weight.shape[0]
    on = (targets >= 0) & (targets < V)
    xs = torch.where(on[:, None], x.double(), torch.zeros((), dtype=torch.float64, device=x.device))
    w = weight.double()
    t = torch.where(on, targets, torch.zeros_like(targets)).long()[:, None]
    s = xs @ w.T * scale
    size = xs.abs() @ w.abs().T * scale
    es = (D + 3) * F * size + 2 * F * s.abs()
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    el = es.max(1).values + (V + 16) * F + 6 * F * lse.abs()
    zero = torch.zeros_like(lse)
    rows = torch.where(on, lse - s.gather(1, t)[:, 0], zero)
    er = torch.where(on, el + es.gather(1, t)[:, 0] + 6 * F * (lse.abs() + s.gather(1, t)[:, 0].abs()), zero)
    g = factor / max(1, int(on.sum())) if mean else factor
    loss = (rows.sum() * g).view(1)
    eloss = (er.sum() * abs(g) + 4 * F * loss.abs()).view(1)
    ds = p.clone()
    ds.scatter_add_(1, t, torch.full(t.shape, -1.0, dtype=torch.float64, device=x.device))
    ds = torch.where(on[:, None], ds * g * scale, torch.zeros_like(ds))
    eds = p * (es + el[:, None] + 4 * F * (s.abs() + lse.abs()[:, None]) + 8 * F) * abs(g * scale) + 3 * F * ds.abs()
    # a target's coefficient is a difference from 1: its last rounding is of a number up to 1
    eds.scatter_add_(1, t, torch.full(t.shape, 2 * F * abs(g * scale), dtype=torch.float64, device=x.device))
    eds = torch.where(on[:, None], eds, torch.zeros_like(eds))
    if x.dtype != torch.float32:
        eds = eds + half_step(x.dtype) * (ds.abs() + eds)
    a = ds.abs() + eds
    dx, dw = ds @ w, ds.T @ xs
    edx = eds @ w.abs() + (V + 6) * F * (a @ w.abs()) + half_step(x.dtype) * dx.abs() * 1.01 + TINY
    edw = eds.T @ xs.abs() + (N + 6) * F * (a.T @ xs.abs()) + TINY
    edw = edw + half_step(grad_dtype) * (dw.abs() + edw)
    edx = edx + half_step(x.dtype) * edx
    return dict(loss=(loss, eloss + TINY), row_loss=(rows, er), dx=(dx, edx), dweight=(dw, edw))
