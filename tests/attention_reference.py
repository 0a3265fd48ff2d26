"""Rotary positions and attention over packed sequences with shared key/value heads, in 64 bits from the definitions, with
bounds on what the library's roundings can come to.  Runs on the CPU or the GPU.

Roundings counted (u = half a step of the storage type, bf16 2^-8; f = 2^-24, half a step of fp32):
  score   a dot product of dh terms and its scaling: (dh + 3) f sum |q k| scale log2 e in the exponent; a probability is off
          by ln 2 times that, by f times its exponent's size (the difference from the row's statistic is rounded
          once), by 4 f of the exponential itself, and (backward) by f |lse| of the stored statistic
  operand bf16: a probability, or dS, is rounded once more, u
  sums    (number of terms + 4) f of the sum of the absolute terms
  result  u of itself
"""
import math

import torch

F = 2.0 ** -24
LOG2E = 1.4426950408889634


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def frequencies(dims, base=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, original=0.0):
    out = []
    for i in range(dims // 2):
        b = base * factor ** (dims / (dims - 2)) if scaling == "base" else base
        f = b ** (-2.0 * i / dims)
        if scaling == "linear":
            f /= factor
        if scaling == "by_parts":
            w = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
            f = f * w + f * (1 - w) / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rotary(x, positions, dims, layout="half", magnitude=1.0, inverse=False, **scaling):
    """(x turned, bound on the error) in 64 bits; x [rows, heads, dh], positions [rows]."""
    y = x.double()
    t = torch.outer(positions.double(), frequencies(dims, **scaling).to(x.device))
    c, s = (torch.cos(t) * magnitude)[:, None], (torch.sin(t) * (-magnitude if inverse else magnitude))[:, None]
    h = dims // 2
    ia, ib = (slice(0, h), slice(h, dims)) if layout == "half" else (slice(0, dims, 2), slice(1, dims, 2))
    a, b = y[..., ia], y[..., ib]
    out = y.clone()
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    # cosine and sine: an angle of at most pi rounded to fp32 (pi f), 64-bit angles of up to 2^32 turns (2^32 2^-52 2 pi, counted with
    # the magnitude of the positions below), the functions' own 2 f, the magnitude's rounding f; two products and a sum: 2 f
    far = positions.abs().double().max().item() * 2.0 ** -51 if len(positions) else 0.0
    size = (a.abs() + b.abs()) * abs(magnitude)
    err = torch.zeros_like(y)
    err[..., ia] = err[..., ib] = size * ((math.pi + 5) * F + far)
    return out, err + half_step(x.dtype) * out.abs() + 1e-38


class Packed:
    """Sequences with lengths lq, lk; q [sum lq, H, dh], k and v [sum lk, K, dh]."""

    def __init__(self, q, k, v, lq, lk, causal, scale=None):
        self.q, self.k, self.v, self.lq, self.lk, self.causal = q, k, v, lq, lk, causal
        self.scale = q.shape[2] ** -0.5 if scale is None else scale
        self.group = q.shape[1] // k.shape[1]
        self.u = half_step(q.dtype)
        self.operand = self.u if q.dtype != torch.float32 else 0.0

    def _pieces(self):
        a = b = 0
        for n, m in zip(self.lq, self.lk):
            for h in range(self.q.shape[1]):
                yield slice(a, a + n), slice(b, b + m), h, h // self.group, n, m
            a, b = a + n, b + m

    def _scores(self, rows, keys, h, hk, n, m):
        q, k = self.q[rows, h].double(), self.k[keys, hk].double()
        s = q @ k.T * self.scale
        off = (q.shape[1] + 3) * F * (q.abs() @ k.abs().T) * self.scale     # (natural logarithm's units)
        unseen = torch.zeros_like(s, dtype=torch.bool)
        if self.causal:
            unseen = torch.arange(m, device=s.device)[None] > torch.arange(n, device=s.device)[:, None] + (m - n)
        return s.masked_fill(unseen, -math.inf), off.masked_fill(unseen, 0.0)

    def forward(self):
        """o, lse and their bounds."""
        N, H, D = self.q.shape
        z = lambda *s, v=0.0: torch.full(s, v, dtype=torch.float64, device=self.q.device)
        o, lse, eo, el = z(N, H, D), z(N, H, v=-math.inf), z(N, H, D), z(N, H)
        for rows, keys, h, hk, n, m in self._pieces():
            if n == 0 or m == 0:
                continue
            s, off = self._scores(rows, keys, h, hk, n, m)
            l = torch.logsumexp(s, 1)
            none = l == -math.inf
            p = torch.exp(s - l.masked_fill(none, 0.0)[:, None])
            v = self.v[keys, hk].double()
            lse[rows, h] = l * LOG2E
            o[rows, h] = p @ v
            span = (s.masked_fill(s == -math.inf, 0.0).abs().amax(1, keepdim=True) * 2 + l.masked_fill(none, 0.0).abs()[:, None]) * LOG2E
            rel = off + F * span + 6 * F                       # of a probability before its rounding
            worst = rel.amax(1, keepdim=True)
            av = v.abs()
            eo[rows, h] = (p * (rel + worst + self.operand)) @ av * 1.01 + (m + 12) * F * (p @ av) + self.u * (p @ v).abs() + 1e-37
            el[rows, h] = (worst[:, 0] + (m + 8) * F) * LOG2E * 1.01 + 3 * F * l.masked_fill(none, 0.0).abs() * LOG2E
        return o, lse, eo, el

    def backward(self, o, lse, do):
        """dq, dk, dv and their bounds; o and lse as the forward pass left them."""
        q, k, v = self.q, self.k, self.v
        new = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)
        dq, dk, dv, eq, ek, ev, cq, ck, cv = new(q), new(k), new(v), new(q), new(k), new(v), new(q), new(k), new(v)
        D, c = q.shape[2], self.scale
        for rows, keys, h, hk, n, m in self._pieces():
            if n == 0 or m == 0:
                continue
            s, off = self._scores(rows, keys, h, hk, n, m)
            l = lse[rows, h].double() / LOG2E
            p = torch.exp(s - torch.where(l == -math.inf, torch.full_like(l, math.inf), l)[:, None])
            g, oo = do[rows, h].double(), o[rows, h].double()
            vv, kk, qq = v[keys, hk].double(), k[keys, hk].double(), q[rows, h].double()
            delta = (g * oo).sum(1, keepdim=True)
            dp = g @ vv.T
            ds = p * (dp - delta)
            dq[rows, h] = ds @ kk * c
            dk[keys, hk] += ds.T @ qq * c
            dv[keys, hk] += p.T @ g
            fin = torch.where(l == -math.inf, torch.zeros_like(l), l).abs()[:, None]
            rel = off + F * (s.masked_fill(s == -math.inf, 0.0).abs() + 2 * fin) * LOG2E + 6 * F
            edp = (D + 4) * F * (g.abs() @ vv.abs().T + (g * oo).abs().sum(1, keepdim=True)) + 2 * F * (dp.abs() + delta.abs())
            eds = (rel + self.operand) * ds.abs() * 1.01 + p * edp
            group = self.group
            cq[rows, h] = (m + 8) * F * (ds.abs() @ kk.abs()) * c
            ck[keys, hk] += (n * group + 8) * F * (ds.abs().T @ qq.abs()) * c
            cv[keys, hk] += (n * group + 8) * F * (p.T @ g.abs())
            eq[rows, h] = eds @ kk.abs() * c
            ek[keys, hk] += eds.T @ qq.abs() * c
            ev[keys, hk] += (p * (rel + self.operand)).T @ g.abs() * 1.01
        out = [e + s + self.u * x.abs() + 1e-37 for e, s, x in ((eq, cq, dq), (ek, ck, dk), (ev, cv, dv))]
        return dq, dk, dv, *out


def assert_within(got, want, bound, tag):
    """Every element of `got` within its own bound of `want` (infinities equal)."""
    g = got.double()
    assert g.shape == want.shape, f"{tag}: {tuple(g.shape)} for {tuple(want.shape)}"
    same = (g == want) | (torch.isnan(g) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(bound), (g - want).abs() / bound)
    off = torch.where(torch.isnan(off), torch.full_like(off, math.inf), off)
    if off.numel() and off.max() > 1.0:
        i = int(off.flatten().argmax())
        raise AssertionError(f"{tag}: element {i} of {tuple(g.shape)} is {g.flatten()[i].item()!r}, should be "
                             f"{want.flatten()[i].item()!r} within {bound.flatten()[i].item():.3g}; {int((off > 1).sum())} are outside")
