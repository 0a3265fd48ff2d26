"""Rotary positions and attention over packed sequences with shared key/value heads on the GPU, element by element against
the definitions in 64 bits (tests/attention_reference.py, which also derives every tolerance from the roundings)."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import attention_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SENTINEL = 12345.0          # a value that no result takes


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def offsets(lens, extra=0):
    off = [extra]
    for n in lens:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int32, device="cuda")


# ---- rotary -------------------------------------------------------------------------------------------------------
def check_rotary(x, out, dims, positions=None, first=0, period=0, inverse=False, layout="half", magnitude=1.0, **scaling):
    rot = B.make_rotary(dims, layout=layout, magnitude=magnitude, **scaling)
    x0 = x.clone()
    B.hbp_rotary(rot, x, out, positions=positions, first=first, period=period, inverse=inverse)
    n = torch.arange(x.shape[0], device="cuda", dtype=torch.int64)
    pos = (first + (n % period if period else n)) if positions is None else positions
    want, bound = R.rotary(x0, pos, dims, layout, magnitude, inverse, **scaling)
    R.assert_within(out, want, bound, "rotary")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,n,dh,dims", [(1, 1, 8, 2), (1, 40, 128, 128), (3, 5, 72, 36), (257, 3, 64, 64), (129, 9, 64, 22),
                                            (100, 2, 128, 32), (33, 7, 96, 48), (65, 1, 256, 256), (17, 6, 40, 40), (1000, 4, 80, 8)])
def test_rotary(rows, n, dh, dims, layout, dtype):
    x = normal((rows, n, dh), TYPES[dtype], rows)
    for inverse in (False, True):
        check_rotary(x, torch.empty_like(x), dims, first=rows, inverse=inverse, layout=layout, magnitude=1.0 if n % 2 else 0.7)


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=8.0), dict(scaling="base", factor=8.0, base=500000.0),
                                     dict(scaling="by_parts", factor=8.0, original=4096.0, low=1.0, high=32.0), dict(base=1.5)])
def test_rotary_scaled_and_far(scaling):
    x = normal((300, 3, 64), torch.float32, 1)
    check_rotary(x, torch.empty_like(x), 64, first=1 << 20, **scaling)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (300,), device="cuda", dtype=torch.int32)
    check_rotary(x, torch.empty_like(x), 64, positions=pos, **scaling)
    check_rotary(x, torch.empty_like(x), 64, first=-5, period=77, **scaling)
    check_rotary(x, torch.empty_like(x), 64, period=1 << 40, **scaling)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dims", [64, 24, 6])
def test_rotary_strided_and_in_place(dims, layout, dtype):
    """Query and key heads side by side in a projection's output, head after head, rows that are read again and again; what
    lies between stays."""
    big = normal((70, 12, 64), TYPES[dtype], 2)
    want = torch.empty((70, 9, 64), dtype=big.dtype, device="cuda")
    check_rotary(big[:, 1:10], want, dims, layout=layout)
    keep = big.clone()
    B.hbp_rotary(B.make_rotary(dims, layout=layout), big[:, 1:10], big[:, 1:10])
    assert torch.equal(big[:, 1:10], want)
    assert torch.equal(big[:, :1], keep[:, :1]) and torch.equal(big[:, 10:], keep[:, 10:])
    heads_first = torch.full((9, 80, 64), SENTINEL, dtype=big.dtype, device="cuda")
    B.hbp_rotary(B.make_rotary(dims, layout=layout), keep[:, 1:10], heads_first.transpose(0, 1)[:70])
    assert torch.equal(heads_first.transpose(0, 1)[:70], want) and bool((heads_first[:, 70:] == SENTINEL).all())
    one = keep[:1, 1:2].expand(70, 9, 64)
    check_rotary(one, torch.empty_like(want), dims, layout=layout)


def test_rotary_of_nothing_and_of_infinities():
    x = torch.empty((0, 4, 64), device="cuda")
    B.hbp_rotary(B.make_rotary(64), x, torch.empty_like(x))
    x = normal((4, 2, 64), torch.float32, 3)
    x[1, 0, 5], x[2, 1, 40] = math.inf, math.nan
    y = torch.empty_like(x)
    B.hbp_rotary(B.make_rotary(64), x, y, first=1)
    want, _ = R.rotary(x, torch.arange(1, 5, device="cuda"), 64)
    assert torch.equal(torch.isfinite(y), torch.isfinite(want))


# ---- attention ----------------------------------------------------------------------------------------------------
def check_attention(q, k, v, lq, lk, causal, do=None, seqs=None, scale=None, tag=""):
    """Forward and backward of one packed problem; returns the Attention."""
    how = dict(seqs=seqs) if seqs else dict(q_offsets=offsets(lq), k_offsets=offsets(lk))
    a = B.make_attention(q, k, v, causal=causal, scale=scale, **how)
    for t in (a.o, a.dq, a.dk, a.dv, a.lse):
        t.fill_(SENTINEL)
    B.hbp_attention_forward(a)
    ref = R.Packed(q, k, v, lq, lk, causal, scale)
    o, lse, eo, el = ref.forward()
    R.assert_within(a.lse, lse, el, tag + " lse")
    R.assert_within(a.o, o, eo, tag + " o")
    if do is not None:
        B.hbp_attention_backward(a, do)
        dq, dk, dv, eq, ek, ev = ref.backward(a.o, a.lse, do)
        R.assert_within(a.dv, dv, ev, tag + " dv")
        R.assert_within(a.dk, dk, ek, tag + " dk")
        R.assert_within(a.dq, dq, eq, tag + " dq")
    return a


def problem(lq, lk, H, K, D, dtype, seed=0):
    n, m = sum(lq), sum(lk)
    return [normal(s, TYPES[dtype], seed + i) for i, s in enumerate(((n, H, D), (m, K, D), (m, K, D), (n, H, D)))]


SELF = [[1], [2], [31], [32], [33], [64], [65], [127], [129], [300], [1, 1, 1, 1], [5, 0, 40, 1, 0, 77], [0, 0, 3], [100, 28, 128, 64],
        [513], [1030]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", SELF, ids=str)
def test_attention_lengths(lens, causal, dtype):
    q, k, v, do = problem(lens, lens, 4, 2, 64, dtype)
    check_attention(q, k, v, lens, lens, causal, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,K", [(1, 1), (3, 3), (8, 1), (6, 2), (7, 1), (12, 4), (64, 1), (40, 1)])
@pytest.mark.parametrize("dh", [64, 128])
def test_attention_heads(H, K, dh, causal, dtype):
    lens = [70, 1, 95]
    q, k, v, do = problem(lens, lens, H, K, dh, dtype, 5)
    check_attention(q, k, v, lens, lens, causal, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [8, 16, 24, 32, 40, 48, 72, 80, 96, 104, 120, 128])
def test_attention_widths(dh, dtype):
    lens = [50, 33, 150]
    q, k, v, do = problem(lens, lens, 4, 2, dh, dtype, 7)
    for causal in (True, False):
        check_attention(q, k, v, lens, lens, causal, do)


# queries and keys of unequal numbers: few over many, many over few (causal: queries that see nothing), none on one side
CROSS = [([1], [1000]), ([1, 1, 1], [7, 300, 65]), ([5], [64]), ([16, 3], [129, 2000]), ([64], [5]), ([130], [1]), ([9, 4], [0, 6]),
         ([0, 4], [5, 9]), ([200], [70]), ([70], [200]), ([2, 300, 40], [300, 2, 40]), ([1], [0]), ([3], [4099]), ([33, 32], [1024, 1025])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", CROSS, ids=str)
def test_attention_unequal_lengths(lq, lk, causal, dtype):
    for H, K, dh in ((4, 2, 64), (8, 1, 128), (2, 2, 40)):
        q, k, v, do = problem(lq, lk, H, K, dh, dtype, 11)
        check_attention(q, k, v, lq, lk, causal, do, tag=f"{H}/{K} x {dh}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_equal_lengths_without_offsets(dtype):
    q, k, v, do = problem([45] * 5, [45] * 5, 6, 3, 64, dtype, 13)
    a = check_attention(q, k, v, [45] * 5, [45] * 5, True, do, seqs=5)
    b = check_attention(q, k, v, [45] * 5, [45] * 5, True, do)
    for x, y in ((a.o, b.o), (a.lse, b.lse), (a.dq, b.dq), (a.dk, b.dk), (a.dv, b.dv)):
        assert torch.equal(x, y)
    q, k, v, do = problem([1] * 3, [130] * 3, 8, 2, 128, dtype, 14)
    check_attention(q, k, v, [1] * 3, [130] * 3, True, do, seqs=3)
    q, k, v, do = problem([0] * 2, [6] * 2, 2, 2, 8, dtype, 15)
    a = check_attention(q, k, v, [0] * 2, [6] * 2, True, do, seqs=2)
    assert not a.dk.any() and not a.dv.any()
    q, k, v, do = problem([6] * 2, [0] * 2, 2, 2, 8, dtype, 16)
    check_attention(q, k, v, [6] * 2, [0] * 2, False, do, seqs=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_many_sequences(dtype):
    lens = [(7 * i) % 13 for i in range(400)]
    q, k, v, do = problem(lens, lens, 2, 1, 32, dtype, 17)
    check_attention(q, k, v, lens, lens, True, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-3, 1.0, 4.0])
def test_attention_scales_and_large_scores(scale, dtype):
    """Scores up to several hundred: rows that are all but one key's; a maximum that grows along the keys."""
    lens = [200, 60]
    q, k, v, do = problem(lens, lens, 4, 2, 64, dtype, 19)
    k[:200] *= torch.linspace(0.1, 2.0, 200, device="cuda")[:, None, None].to(k.dtype)
    check_attention(q, k, v, lens, lens, True, do, scale=scale)
    check_attention(q, -k, v, lens, lens, False, do, scale=scale)


def strided(t, how):
    """The same values elsewhere: side by side with others in wider rows, or head after head with rows between."""
    n, h, d = t.shape
    if how == "rows":
        big = torch.full((n, h + 3, d + 8), SENTINEL, dtype=t.dtype, device="cuda")
        view = big[:, 1:1 + h, :d]
    else:
        big = torch.full((h, n + 2, d), SENTINEL, dtype=t.dtype, device="cuda")
        view = big[:, 1:1 + n].transpose(0, 1)
    view.copy_(t)
    return big, view


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["rows", "heads"])
@pytest.mark.parametrize("dh", [64, 96])
def test_attention_strides(dh, how, dtype):
    lens = [37, 0, 130]
    q, k, v, do = problem(lens, lens, 6, 2, dh, dtype, 23)
    a = check_attention(q, k, v, lens, lens, True, do)
    (_, q2), (_, k2), (_, v2), (_, do2) = (strided(t, how) for t in (q, k, v, do))
    b = B.make_attention(q2, k2, v2, q_offsets=a.q_offsets, k_offsets=a.k_offsets)
    outs = {}
    for name in ("o", "dq", "dk", "dv"):
        big, view = strided(torch.full_like(getattr(a, name), SENTINEL), how)
        setattr(b, name, view)
        outs[name] = (big, view)
    B.hbp_attention_forward(b)
    B.hbp_attention_backward(b, do2)
    assert torch.equal(a.lse, b.lse)
    for name, (big, view) in outs.items():
        assert torch.equal(getattr(a, name), view), name
        view.fill_(SENTINEL)
        assert bool((big == SENTINEL).all()), f"{name}: written outside"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_leaves_rows_outside_the_sequences(dtype):
    q, k, v, do = problem([100], [90], 4, 2, 64, dtype, 29)
    lq, lk = [30, 41], [50, 21]
    a = B.make_attention(q, k, v, q_offsets=offsets(lq, 7), k_offsets=offsets(lk, 9))
    for t in (a.o, a.dq, a.dk, a.dv, a.lse):
        t.fill_(SENTINEL)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    sq, sk = slice(7, 78), slice(9, 80)
    ref = R.Packed(q[sq], k[sk], v[sk], lq, lk, True)
    o, lse, eo, el = ref.forward()
    R.assert_within(a.o[sq], o, eo, "o")
    for got, want, bound in zip((a.dq[sq], a.dk[sk], a.dv[sk]), *[ref.backward(a.o[sq], a.lse[sq], do[sq])[i:i + 3] for i in (0, 3)]):
        R.assert_within(got, want, bound, "gradient")
    for t, s in ((a.o, sq), (a.dq, sq), (a.lse, sq), (a.dk, sk), (a.dv, sk)):
        assert bool((t[:s.start] == SENTINEL).all()) and bool((t[s.stop:] == SENTINEL).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_offsets_past_the_rows_are_cut(dtype):
    q, k, v, do = problem([50], [50], 2, 1, 64, dtype, 31)
    a = B.make_attention(q, k, v, q_offsets=torch.tensor([-5, 20, 1000], dtype=torch.int32, device="cuda"),
                         k_offsets=torch.tensor([-1, 20, 51], dtype=torch.int32, device="cuda"))
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    b = check_attention(q, k, v, [20, 30], [20, 30], True, do)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_attention_infinities_and_nans_reach_what_sees_them(bad, dh, dtype):
    """One bad value, one bad key, one bad query in the first of two sequences, at the first key head: what does not see it is
    what it is without.  (A bad value reaches one channel of o, and no dv.)"""
    lens = [150, 40]
    q, k, v, do = problem(lens, lens, 4, 2, dh, dtype, 37)
    clean = check_attention(q, k, v, lens, lens, True, do)
    ref = R.Packed(q, k, v, lens, lens, True)
    o, lse, eo, el = ref.forward()
    dq, dk, dv, eq, ek, ev = ref.backward(clean.o, clean.lse, do)
    eq, ek, ev = (2 * e for e in (eq, ek, ev))             # (of gradients from this call's own o and lse)
    for name, row in (("v", 100), ("k", 100), ("q", 20)):
        t = dict(q=q.clone(), k=k.clone(), v=v.clone())
        t[name][row, 0, 3] = bad
        a = B.make_attention(t["q"], t["k"], t["v"], q_offsets=clean.q_offsets, k_offsets=clean.k_offsets)
        B.hbp_attention_forward(a)
        B.hbp_attention_backward(a, do)
        rows = torch.zeros((190, 4), dtype=torch.bool, device="cuda")       # (query, head) that sees it
        keys = torch.zeros((190, 2), dtype=torch.bool, device="cuda")       # (key, key head) that such a query sees
        if name == "q":
            rows[20, 0], keys[:21, 0] = True, True
        else:
            rows[100:150, :2], keys[:150, 0] = True, True
        R.assert_within(a.o[~rows], o[~rows], eo[~rows], name + " o")
        R.assert_within(a.dq[~rows], dq[~rows], eq[~rows], name + " dq")
        R.assert_within(a.dk[~keys], dk[~keys], ek[~keys], name + " dk")
        R.assert_within(a.dv[~keys], dv[~keys], ev[~keys], name + " dv")
        if name == "v":
            other = [c for c in range(dh) if c != 3]
            R.assert_within(a.o[..., other], o[..., other], eo[..., other], "v o, other channels")
            R.assert_within(a.lse, lse, el, "v lse")
            R.assert_within(a.dv, dv, ev, "v dv")
            assert not torch.isfinite(a.o[rows][:, 3]).any()
        if name == "q" or (name == "k" and bad != bad):
            assert not torch.isfinite(a.o[rows]).any()


def test_attention_rows_of_minus_infinity_scores_weigh_nothing():
    q, k, v, do = problem([40], [40], 2, 1, 64, "bf16", 41)
    q[:, :, 0] = 1.0
    k[:10, 0, 0] = -math.inf                               # the first ten keys score minus infinity
    a = B.make_attention(q, k, v)
    B.hbp_attention_forward(a)
    assert bool((a.lse[:10] == -math.inf).all()) and not a.o[:10].any()
    ref = R.Packed(q, k, v, [40], [40], True)
    o, lse, eo, el = ref.forward()
    assert torch.isfinite(a.o).all() and torch.isfinite(a.lse[10:]).all()
    eo = torch.where(torch.isfinite(eo), eo, torch.full_like(eo, 2.0 ** -7))
    R.assert_within(a.o[10:], o[10:], eo[10:] + 2.0 ** -7 * v.double().abs().max(), "o")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lq,lk", [([300, 20], [300, 20]), ([1, 2], [2500, 700])], ids=str)
def test_attention_is_repeatable(lq, lk, dtype):
    q, k, v, do = problem(lq, lk, 8, 2, 64, dtype, 43)
    a = check_attention(q, k, v, lq, lk, True, do)
    first = [t.clone() for t in (a.o, a.lse, a.dq, a.dk, a.dv)]
    for _ in range(3):
        a.workspace.random_(0, 255)                        # nothing is kept in it from one call to the next
        B.hbp_attention_forward(a)
        B.hbp_attention_backward(a, do)
        for x, y in zip(first, (a.o, a.lse, a.dq, a.dk, a.dv)):
            assert torch.equal(x, y)


def chain(rot, qkv, turned, a, do, dturned, dqkv, H, K):
    B.hbp_rotary(rot, qkv[:, :H + K], turned, period=64)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    B.hbp_rotary(rot, dturned, dqkv[:, :H + K], period=64, inverse=True)


def make_chain(dtype, seed, lens=(64, 64, 64), H=6, K=2, D=64):
    n = sum(lens)
    qkv, do = normal((n, H + 2 * K, D), TYPES[dtype], seed), normal((n, H, D), TYPES[dtype], seed + 1)
    turned, dqkv = torch.empty_like(qkv[:, :H + K].contiguous()), torch.empty_like(qkv)
    dturned = torch.empty_like(turned)
    a = B.make_attention(turned[:, :H], turned[:, H:], qkv[:, H + K:], seqs=len(lens))
    a.dq, a.dk, a.dv = dturned[:, :H], dturned[:, H:], dqkv[:, H + K:]
    return B.make_rotary(D), qkv, turned, a, do, dturned, dqkv, H, K


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_positions_attention_and_their_gradient_together(dtype):
    """A layer's share: each step against the definition on what the step before left."""
    c = make_chain(dtype, 47)
    chain(*c)
    rot, qkv, turned, a, do, dturned, dqkv, H, K = c
    pos = torch.arange(192, device="cuda") % 64
    R.assert_within(turned, *R.rotary(qkv[:, :H + K], pos, 64), "turned")
    ref = R.Packed(turned[:, :H], turned[:, H:], qkv[:, H + K:], [64] * 3, [64] * 3, True)
    o, lse, eo, el = ref.forward()
    R.assert_within(a.o, o, eo, "o")
    dq, dk, dv, eq, ek, ev = ref.backward(a.o, a.lse, do)
    R.assert_within(dturned, torch.cat((dq, dk), 1), torch.cat((eq, ek), 1), "dq, dk")
    R.assert_within(dqkv[:, H + K:], dv, ev, "dv")
    R.assert_within(dqkv[:, :H + K], *R.rotary(dturned, pos, 64, inverse=True), "turned back")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    """The whole run in a graph, replayed between eager work on other data, against the eager result every time."""
    c, other = make_chain(dtype, 53), make_chain(dtype, 59, lens=(64, 64, 64, 64, 64))
    chain(*c)
    torch.cuda.synchronize()
    want = [c[3].o.clone(), c[6].clone()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        chain(*c)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(*c)
    for i in range(4):
        c[3].o.zero_()
        c[6].zero_()
        graph.replay()
        chain(*other)
        torch.cuda.synchronize()
        assert torch.equal(c[3].o, want[0]) and torch.equal(c[6], want[1]), f"replay {i}"


def test_two_streams_at_once():
    """Two calls with workspaces of their own, on two streams at once."""
    chains = [make_chain("bf16", 61, lens=[64] * 40), make_chain("bf16", 67, lens=[64] * 40)]
    wants = []
    for c in chains:
        chain(*c)
        torch.cuda.synchronize()
        wants.append((c[3].o.clone(), c[6].clone()))
    streams = [torch.cuda.Stream() for _ in chains]
    for _ in range(5):
        for c, s in zip(chains, streams):
            with torch.cuda.stream(s):
                chain(*c)
    torch.cuda.synchronize()
    for c, w in zip(chains, wants):
        assert torch.equal(c[3].o, w[0]) and torch.equal(c[6], w[1])


def test_a_stream_given_by_its_handle():
    s = torch.cuda.Stream()
    x = normal((300, 4, 64), torch.bfloat16, 71)
    y, z = torch.empty_like(x), torch.empty_like(x)
    torch.cuda.synchronize()
    B.hbp_rotary(B.make_rotary(64), x, y, stream=s.cuda_stream)
    s.synchronize()
    B.hbp_rotary(B.make_rotary(64), x, z)
    assert torch.equal(y, z)


# Every form of the kernels by its sizes: wavefronts by themselves, workgroups of many rows, of few, shares (both sides), ragged or not.
FORMS = [([60 + i % 9 for i in range(60)], None, 8, 8), ([3, 0, 64, 65, 1, 100, 33] * 20, None, 8, 4), ([256] * 20, None, 16, 8),
         ([1] * 150, [200 + i % 100 for i in range(150)], 8, 8), ([1] * 40, [1000] * 40, 32, 32), ([1500, 900], None, 16, 2),
         ([700] * 12, None, 12, 6), ([2000], None, 4, 1), ([5], [6000], 8, 8), ([900], [40], 8, 8), ([40, 2], [3000, 100], 4, 4),
         ([64] * 70, None, 8, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lq,lk,H,K", FORMS, ids=[f"{len(f[0])}x{f[0][0]}" for f in FORMS])
def test_attention_forms(lq, lk, H, K, dh, dtype):
    lk = lq if lk is None else lk
    if len(lq) * max(lq) * max(lk) * H * dh > 3e10:        # (the reference's time)
        H, K = H // K, 1
    q, k, v, do = problem(lq, lk, H, K, dh, dtype, 73)
    for causal in (True, False):
        check_attention(q, k, v, lq, lk, causal, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,K", [([64] * 70, 8, 8), ([600] * 2, 4, 4), ([1030], 4, 2)])
def test_infinities_in_every_form(lens, H, K, dtype):
    """A bad value at the last key of the first sequence: its earlier queries, and every other sequence, are as without it."""
    q, k, v, do = problem(lens, lens, H, K, 64, dtype, 79)
    clean = check_attention(q, k, v, lens, lens, True, do)
    n = lens[0]
    bad = v.clone()
    bad[n - 1, :, 5] = math.nan
    a = B.make_attention(q, k, bad, q_offsets=clean.q_offsets, k_offsets=clean.k_offsets)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    seen = torch.zeros(sum(lens), dtype=torch.bool, device="cuda")
    seen[n - 1] = True
    for name in ("o", "dq"):
        assert torch.isfinite(getattr(a, name)[~seen]).all(), name
        assert not torch.isfinite(getattr(a, name)[seen]).all(), name
    ref = R.Packed(q, k, v, lens, lens, True)
    o, lse, eo, el = ref.forward()
    R.assert_within(a.lse, lse, el, "lse")
    R.assert_within(a.o[~seen], o[~seen], eo[~seen], "o")
    dq, dk, dv, eq, ek, ev = ref.backward(clean.o, clean.lse, do)
    R.assert_within(a.dq[~seen], dq[~seen], 2 * eq[~seen], "dq")
    R.assert_within(a.dv, dv, ev, "dv")                    # (a value does not enter dv)
    R.assert_within(a.dk[n:], dk[n:], 2 * ek[n:], "dk")


BIG = [([70] * 2, [250] * 2, 2, 2), ([64] * 70, None, 8, 8), ([600] * 5, None, 48, 24), ([1030], None, 4, 2), ([3], [6000], 8, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,H,K", BIG, ids=[f"{len(f[0])}x{f[0][0]}" for f in BIG])
def test_scores_beyond_the_exponents_steps(lq, lk, H, K, causal, dtype):
    """Scores of up to 2^46, of which fp32 keeps steps of 2^23: no two of a head's are closer than 2^33, so that every row is the
    value of the key with its largest score.  q holds 2^20, k the score's two parts (exact in either type), and so are the
    products.  Roundings: lse that of log2 e, of its product and of the difference from 0, 4 f; o where the weight 2^r of the one
    key is rounded to bf16 and divided by its sum: u each for weight and result, and 8 f for fp32's exponential, sum,
    reciprocal and products."""
    lk = lq if lk is None else lk
    g = torch.Generator(device="cuda").manual_seed(83)
    N, M = sum(lq), sum(lk)
    q = torch.zeros((N, H, 64), dtype=TYPES[dtype], device="cuda")
    q[:, :, 0] = q[:, :, 1] = 2.0 ** 20
    place = torch.stack([torch.cat([torch.randperm(n, generator=g, device="cuda") for n in lk]) for _ in range(K)], 1)     # [M, K]
    k = torch.zeros((M, K, 64), dtype=TYPES[dtype], device="cuda")
    k[:, :, 0], k[:, :, 1] = (place // 128) * 2.0 ** 20, (place % 128) * 2.0 ** 13
    v = normal((M, K, 64), TYPES[dtype], 84)
    a = B.make_attention(q, k, v, causal=causal, scale=1.0, q_offsets=offsets(lq), k_offsets=offsets(lk))
    B.hbp_attention_forward(a)
    u = 0.0 if dtype == "f32" else R.half_step(TYPES[dtype])
    r0 = k0 = 0
    for n, m in zip(lq, lk):
        s = place[k0:k0 + m].T[:, None].expand(K, n, m).clone()
        if causal:
            s[:, torch.arange(m, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + (m - n)] = -1
        top, key = s.max(2)                                # [K, n]
        want = v[k0 + key, torch.arange(K, device="cuda")[:, None]].transpose(0, 1).repeat_interleave(H // K, 1).double()
        lse = (top.double() * 2.0 ** 33 * R.LOG2E).T.repeat_interleave(H // K, 1)
        R.assert_within(a.o[r0:r0 + n], want, want.abs() * (2 * u + 8 * R.F) + 1e-38, "o")
        R.assert_within(a.lse[r0:r0 + n], lse, lse.abs() * 4 * R.F + 1e-38, "lse")
        r0, k0 = r0 + n, k0 + m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lq,lk,H,K", BIG, ids=[f"{len(f[0])}x{f[0][0]}" for f in BIG])
def test_nan_throughout(lq, lk, H, K, dtype):
    """What diverged stays so, in every element that sees something."""
    lk = lq if lk is None else lk
    q, k, v, do = (torch.full_like(t, math.nan) for t in problem(lq, lk, H, K, 96, dtype, 89))
    a = B.make_attention(q, k, v, causal=False, q_offsets=offsets(lq), k_offsets=offsets(lk))
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.isnan(getattr(a, name)).all(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,K", [([300] * 2, 3, 1), ([64] * 70, 8, 8)])
def test_rows_computed_once_more_are_repeatable(lens, H, K, dtype):
    """An infinity in one channel of the last key's value: causal rows that do not see it meet it in a tile all the same."""
    q, k, v, do = problem(lens, lens, H, K, 128, dtype, 97)
    v[lens[0] - 1, :, 70] = math.inf
    a = B.make_attention(q, k, v, q_offsets=offsets(lens), k_offsets=offsets(lens))
    bits = torch.int32 if dtype == "f32" else torch.int16
    first = None
    for _ in range(6):
        B.hbp_attention_forward(a)
        B.hbp_attention_backward(a, do)
        now = [getattr(a, name).clone().view(bits) for name in ("o", "dq", "dk", "dv")] + [a.lse.clone().view(torch.int32)]
        assert first is None or all(torch.equal(x, y) for x, y in zip(first, now))
        first = now


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[i % 4 for i in range(3000)], [(7 * i) % 40 for i in range(300)], [0] * 200 + [300, 1] + [0] * 100,
                                  [(i * i) % 90 for i in range(129)], [0] * 140], ids=lambda n: f"{len(n)}of{max(n)}")
def test_attention_hundreds_and_thousands_of_sequences(lens, dtype):
    """Some of them against the definitions, and that every row was written; empty ones between."""
    q, k, v, do = problem(lens, lens, 4, 2, 64, dtype, 101)
    a = B.make_attention(q, k, v, q_offsets=offsets(lens), k_offsets=offsets(lens))
    for t in (a.o, a.dq, a.dk, a.dv, a.lse):
        t.fill_(SENTINEL)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    at, first = 0, []
    for n in lens:
        first.append(at)
        at += n
    some = [i for i, n in enumerate(lens) if n][:: max(1, len(lens) // 80)]
    for i in some:
        n, r = lens[i], slice(first[i], first[i] + lens[i])
        ref = R.Packed(q[r], k[r], v[r], [n], [n], True)
        o, lse, eo, el = ref.forward()
        R.assert_within(a.lse[r], lse, el, "lse")
        R.assert_within(a.o[r], o, eo, "o")
        dq, dk, dv, eq, ek, ev = ref.backward(a.o[r], a.lse[r], do[r])
        R.assert_within(a.dv[r], dv, ev, "dv")
        R.assert_within(a.dk[r], dk, ek, "dk")
        R.assert_within(a.dq[r], dq, eq, "dq")
    for t in (a.o, a.dq, a.dk, a.dv, a.lse):
        assert not (t == SENTINEL).any()                   # every row belongs to a sequence


# many rows of wide heads: 64 for a wavefront
TALL = [([1030] * 12, None, 16, 16), ([290 + i % 21 for i in range(20)], None, 32, 8), ([300] * 20, [340] * 20, 32, 8),
        ([513] * 22, [9] * 22, 16, 8)]


@pytest.mark.parametrize("dh", [72, 96, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,H,K", TALL, ids=[f"{len(f[0])}x{f[0][0]}" for f in TALL])
def test_attention_many_rows_of_wide_heads(lq, lk, H, K, causal, dh):
    lk = lq if lk is None else lk
    q, k, v, do = problem(lq, lk, H, K, dh, "bf16", 103)
    check_attention(q, k, v, lq, lk, causal, do)


def test_many_rows_of_wide_heads_with_infinities_and_large_scores():
    """A NaN in the last key's value reaches the queries that see it alone; scores beyond 2^31 (see above) take their key's value."""
    lens = [300] * 20
    q, k, v, _ = problem(lens, lens, 32, 8, 128, "bf16", 107)
    v[299, :, 100] = math.nan
    a = B.make_attention(q, k, v, q_offsets=offsets(lens), k_offsets=offsets(lens))
    B.hbp_attention_forward(a)
    clean = v.clone()
    clean[299] = 0
    o, lse, eo, el = R.Packed(q, k, clean, lens, lens, True).forward()
    seen = torch.zeros(sum(lens), dtype=torch.bool, device="cuda")
    seen[299] = True
    R.assert_within(a.o[~seen], o[~seen], eo[~seen], "o")
    R.assert_within(a.lse, lse, el, "lse")
    assert torch.isnan(a.o[299, :, 100]).all()
    q.zero_(), k.zero_()
    q[:, :, 0] = 2.0 ** 20
    place = torch.randperm(256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(109))
    k[:, :, 0] = torch.cat([place, place[:44] * 0])[:300].repeat(20)[:, None] * 2.0 ** 20
    B.hbp_attention_forward(a)
    key = torch.cummax(torch.cat([place, place[:44] * 0]), 0).indices.repeat(20) + 300 * torch.arange(20, device="cuda").repeat_interleave(300)
    want = v[key].repeat_interleave(4, 1)
    ok = ~torch.isnan(want)
    ok[299] = False
    assert torch.equal(a.o[ok], want[ok])
