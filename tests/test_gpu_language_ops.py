"""Dropout, embedding and cross entropy on the GPU, element by element against the definitions in 64 bits
(tests/language_reference.py, which also derives every tolerance from the roundings)."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SENTINEL = 12345.0          # a value that no result takes


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def some_tokens(n, vocab, seed, padding=0.1):
    """Few tokens often, as in text; some outside the vocabulary on either side."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    t = (u * math.log(vocab + 1)).exp().floor().long().clamp_(1, vocab) - 1
    out = torch.rand(n, generator=g, device="cuda")
    t[out < padding] = -1
    t[out < padding / 2] = vocab
    return t.to(torch.int32)


# ---- dropout ------------------------------------------------------------------------------------------------------
def check_dropout(x, out, drop, residual=None):
    x0, r0 = x.clone(), None if residual is None else residual.clone()
    B.hbp_dropout(B.make_dropout(*drop), x, out, residual=residual)
    R.assert_within(out, *R.dropout(x0, drop, r0), "dropout")
    if residual is None:
        assert torch.equal(out == 0, (R.multipliers(*x.shape, drop, "cuda") == 0) | (x0 == 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(1, 8), (1, 65536), (3, 72), (257, 64), (1000, 264), (33, 4096), (4099, 512)])
def test_dropout(rows, width, dtype):
    x = normal((rows, width), TYPES[dtype], rows)
    for drop in ((0.1, 3, 0), (0.5, 2 ** 64 - 1, 2 ** 64 - 1), (0.0, 0, 0), (0.9999, 1 << 40, 1 << 33)):
        check_dropout(x, torch.empty_like(x), drop)
    check_dropout(x, torch.empty_like(x), (0.3, 5, 6), residual=normal((rows, width), TYPES[dtype], 7))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_strided_in_place_and_of_infinities(dtype):
    big = normal((70, 96), TYPES[dtype], 2)
    want = torch.empty((70, 64), dtype=big.dtype, device="cuda")
    check_dropout(big[:, 16:80], want, (0.2, 9, 1))
    one = big[:1, :64].expand(70, 64)
    check_dropout(one, torch.empty_like(want), (0.2, 9, 1), residual=big[:, 32:96])
    keep = big.clone()
    B.hbp_dropout(B.make_dropout(0.2, 9, 1), big[:, 16:80], big[:, 16:80])
    assert torch.equal(big[:, 16:80], want) and torch.equal(big[:, :16], keep[:, :16]) and torch.equal(big[:, 80:], keep[:, 80:])
    r, x = keep[:, 16:80].clone(), normal((70, 64), TYPES[dtype], 3)
    ref, bound = R.dropout(x, (0.2, 9, 1), r)
    B.hbp_dropout(B.make_dropout(0.2, 9, 1), x, r, residual=r)
    R.assert_within(r, ref, bound, "onto the residual")
    x[3] = math.inf
    x[4] = math.nan
    out = torch.empty_like(x)
    B.hbp_dropout(B.make_dropout(0.5, 1), x, out)
    stays = R.kept(70, 64, 0.5, 1).cuda()
    assert torch.equal(torch.isfinite(out[3:5]), ~stays[3:5]) and bool((out[3:5][~stays[3:5]] == 0).all())
    B.hbp_dropout(B.make_dropout(0.5, 1), x[:0], out[:0])


def test_dropout_makes_the_same_mask_again_and_others_for_others():
    x = torch.ones((300, 512), device="cuda")
    outs = []
    for seed, offset, counter in ((1, 2, None), (1, 2, None), (1, 3, None), (2, 2, None), (1, 0, 2), (1, 2 ** 64 - 1, 3)):
        out = torch.empty_like(x)
        c = None if counter is None else torch.tensor([counter], dtype=torch.int64, device="cuda")
        B.hbp_dropout(B.make_dropout(0.25, seed, offset, c), x, out)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[4]) and torch.equal(outs[0], outs[5])
    for other in outs[2:4]:
        both = ((outs[0] > 0) & (other > 0)).double().mean().item()
        assert abs(both - 0.5625) < 5 * math.sqrt(0.5625 * 0.4375 / x.numel())               # independent: 0.75 squared
    # eight elements on, a row on: as independent
    k = outs[0] > 0
    for a, b in ((k[:, 8:], k[:, :-8]), (k[1:], k[:-1]), (k[:, 1:], k[:, :-1])):
        assert abs((a & b).double().mean().item() - 0.5625) < 5 * math.sqrt(0.5625 * 0.4375 / a.numel())


# ---- embedding ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", [(1, 1, 8), (1, 50, 64), (37, 9, 72), (300, 1009, 264), (5000, 700, 128), (2100, 20000, 1032)])
def test_embedding_forward(n, vocab, width, dtype):
    table = normal((vocab, width), TYPES[dtype], 1)
    tokens = some_tokens(n, vocab, n)
    for scale, drop in ((1.0, None), (math.sqrt(width), (0.1, 4, 5)), (-0.3, (0.0, 0, 0))):
        e = B.make_embedding(tokens, table, scale=scale, dropout=None if drop is None else B.make_dropout(*drop), grad=False)
        B.hbp_embedding_forward(e)
        R.assert_within(e.out, *R.embedding(tokens, table, scale, drop), "embedding")


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,vocab,width", [(1, 1, 8), (1, 300, 64), (63, 5, 72), (64, 1, 16), (65, 2, 8), (300, 1009, 264), (2047, 17, 128),
                                           (2049, 511, 64), (5000, 70000, 72), (2100, 20000, 520), (20000, 300, 1032), (4096, 263000, 8)])
def test_embedding_backward(n, vocab, width, dtype, grad):
    table = normal((vocab, width), TYPES[dtype], 1)
    tokens, dout = some_tokens(n, vocab, n), normal((n, width), TYPES[dtype], 2)
    for scale, drop in ((1.0, None), (2.5, (0.3, 4, 5))):
        e = B.make_embedding(tokens, table, scale=scale, dropout=None if drop is None else B.make_dropout(*drop),
                             dtable=torch.full((vocab, width), SENTINEL, dtype=TYPES[grad], device="cuda"))
        B.hbp_embedding_backward(e, dout)
        R.assert_within(e.dtable, *R.embedding_grad(tokens, dout, vocab, scale, drop, TYPES[grad]), "dtable")
        first = e.dtable.clone()
        B.hbp_embedding_backward(e, dout)
        assert torch.equal(first, e.dtable)                # bit by bit
        e.dtable = normal((vocab, width), TYPES[grad], 9)
        old = e.dtable.clone()
        B.hbp_embedding_backward(e, dout, accumulate=True)
        R.assert_within(e.dtable, *R.embedding_grad(tokens, dout, vocab, scale, drop, TYPES[grad], old), "accumulated")


@pytest.mark.parametrize("n", [1, 64, 1000, 3000, 200000])
def test_embedding_backward_of_one_token_and_of_none(n):
    """Every row the same token: the longest sums; every row padding; and sums that cancel."""
    dout = normal((n, 64), torch.bfloat16, 3)
    table = normal((500, 64), torch.bfloat16, 4)
    for v in (0, 499, 77, -1, 500):
        tokens = torch.full((n,), v, dtype=torch.int32, device="cuda")
        e = B.make_embedding(tokens, table)
        B.hbp_embedding_backward(e, dout)
        R.assert_within(e.dtable, *R.embedding_grad(tokens, dout, 500, 1.0, None, torch.float32), f"token {v}")


def test_embedding_strides_rows_behind_and_nothing():
    big = normal((40, 200), torch.float32, 5)
    table, tokens = big[:, 8:136], some_tokens(70, 40, 6)
    room = torch.full((80, 256), SENTINEL, device="cuda")
    e = B.make_embedding(tokens, table, out=room[:70, 64:192])
    B.hbp_embedding_forward(e)
    R.assert_within(room[:70, 64:192], *R.embedding(tokens, table, 1.0), "strided")
    assert bool((room[70:] == SENTINEL).all()) and bool((room[:, :64] == SENTINEL).all()) and bool((room[:, 192:] == SENTINEL).all())
    grad = torch.full((50, 160), SENTINEL, device="cuda")
    d = normal((70, 300), torch.float32, 7)[:, 100:228]
    d = torch.as_strided(normal((70, 304), torch.float32, 7), (70, 128), (304, 1), 96)
    e = B.make_embedding(tokens, table, dtable=grad[:40, :128])
    B.hbp_embedding_backward(e, d)
    R.assert_within(grad[:40, :128], *R.embedding_grad(tokens, d, 40, 1.0, None, torch.float32), "strided gradient")
    assert bool((grad[40:] == SENTINEL).all()) and bool((grad[:, 128:] == SENTINEL).all())
    one = d[:1].expand(70, 128)
    B.hbp_embedding_backward(e, one)
    R.assert_within(grad[:40, :128], *R.embedding_grad(tokens, one, 40, 1.0, None, torch.float32), "one row again and again")
    none = tokens[:0]
    e = B.make_embedding(none, table)
    B.hbp_embedding_forward(e)
    B.hbp_embedding_backward(e, d[:0])
    assert bool((e.dtable == 0).all())
    e.dtable.fill_(3.0)
    B.hbp_embedding_backward(e, d[:0], accumulate=True)
    assert bool((e.dtable == 3).all())


def test_embedding_infinities_reach_their_rows_only():
    table = normal((30, 64), torch.bfloat16, 8)
    table[4], table[5] = math.inf, math.nan
    tokens = torch.tensor([4, 5, 6, -1, 30, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    e = B.make_embedding(tokens, table)
    B.hbp_embedding_forward(e)
    assert torch.isfinite(e.out.float()).all(1).tolist() == [False, False, True, True, True, True, True] and bool((e.out[3:] == 0).all())
    d = normal((7, 64), torch.bfloat16, 9)
    d[0], d[3], d[5] = math.nan, math.inf, math.nan
    B.hbp_embedding_backward(e, d)
    fine = torch.isfinite(e.dtable).all(1)
    assert not bool(fine[4]) and int(fine.sum()) == 29


# ---- cross entropy ------------------------------------------------------------------------------------------------
def check_loss(x, w, t, scale=1.0, mean=True, factor=1.0, grad=torch.float32, again=True, **out):
    want = R.cross_entropy(x, w, t, scale, mean, factor, grad)
    c = B.make_cross_entropy(x, w, t, scale=scale, mean=mean, factor=factor, **dict(dict(dweight=torch.empty(w.shape, dtype=grad, device="cuda")), **out))
    B.hbp_loss_cross_entropy(c)
    for name, (value, bound) in want.items():
        R.assert_within(getattr(c, name), value, bound, name)
    alone = B.make_cross_entropy(x, w, t, scale=scale, mean=mean, factor=factor, grad=False)
    B.hbp_loss_cross_entropy(alone)
    R.assert_within(alone.loss, *want["loss"], "the loss alone")
    R.assert_within(alone.row_loss, *want["row_loss"], "row losses alone")
    if again:
        keep = [v.clone() for v in (c.loss, c.row_loss, c.dx, c.dweight)]
        c.workspace.fill_(255)                             # (NaN in every type: nothing of the last call is read)
        B.hbp_loss_cross_entropy(c)
        assert all(torch.equal(a, b) for a, b in zip(keep, (c.loss, c.row_loss, c.dx, c.dweight)))      # bit by bit
    return c


SIZES = [(1, 1, 8), (1, 50, 16), (2, 9, 8), (8, 2000, 256), (3, 257, 72), (70, 4096, 64), (333, 1009, 72), (130, 70, 264), (257, 1000, 128),
         (64, 513, 1032), (1000, 300, 512), (2000, 70, 128), (40, 3000, 8)]


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_cross_entropy(n, vocab, width, dtype, grad):
    x, w = normal((n, width), TYPES[dtype], n), normal((vocab, width), TYPES[dtype], 2, 2.0 / math.sqrt(width))
    t = some_tokens(n, vocab, 3, padding=0.2 if n > 2 else 0.0)
    check_loss(x, w, t, grad=TYPES[grad])
    check_loss(x, w, t, scale=0.3, mean=False, factor=-1.5, grad=TYPES[grad])


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", [(1000, 9300, 128), (1000, 9300, 160), (4101, 2381, 256), (4090, 9300, 1024), (8192, 1100, 256), (2048, 9216, 264), (900, 20001, 512), (1000, 9300, 72), (1000, 9300, 1000),
                                           (4090, 9300, 904), (250, 40100, 776), (600, 20001, 264),
                                           (8190, 5003, 1024)])
def test_cross_entropy_of_many_tiles(n, vocab, width, grad):
    """Sizes whose logits meet no memory: whole tiles, tiles and a rest, contractions that are no multiple of 64, rows filled up."""
    x, w = normal((n, width), torch.bfloat16, n), normal((vocab, width), torch.bfloat16, 2, 2.0 / math.sqrt(width))
    t = some_tokens(n, vocab, 3)
    t[5], t[6], t[7] = vocab - 1, vocab // 256 * 256, vocab // 256 * 256 - 1
    check_loss(x, w, t, grad=TYPES[grad])
    check_loss(x, w, t, scale=0.5, mean=False, factor=-0.25, grad=TYPES[grad], again=False)


def test_cross_entropy_of_many_tiles_in_pieces():
    n, vocab, width = 16384, 33100, 128
    x, w = normal((n, width), torch.bfloat16, n), normal((vocab, width), torch.bfloat16, 2, 2.0 / math.sqrt(width))
    check_loss(x, w, some_tokens(n, vocab, 3))


def test_cross_entropy_of_many_tiles_infinities():
    n, vocab, width = 1000, 9300, 128
    x, w = normal((n, width), torch.bfloat16, 1), normal((vocab, width), torch.bfloat16, 2)
    t = some_tokens(n, vocab, 3, padding=0.5)
    out = (t < 0) | (t >= vocab)
    clean = check_loss(x, w, t)
    x[out] = math.nan
    c = B.make_cross_entropy(x, w, t)
    B.hbp_loss_cross_entropy(c)
    for name in ("loss", "row_loss", "dx", "dweight"):
        assert torch.equal(getattr(c, name), getattr(clean, name)), name
    bad = (~out).nonzero()[:2, 0]
    x[bad[0], 5], x[bad[1], 6] = math.nan, math.inf
    B.hbp_loss_cross_entropy(c)
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[bad] = False
    assert torch.equal(torch.isfinite(c.row_loss), fine) and torch.equal(torch.isfinite(c.dx.float()).all(1), fine)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cross_entropy_of_a_vocabulary_in_pieces(dtype):
    """Few rows, more weights than a piece takes."""
    n, vocab, width = 5, (1 << 20) + 300, 8
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2)
    t = torch.tensor([0, (1 << 20) - 1, 1 << 20, vocab - 1, -1], dtype=torch.int32, device="cuda")
    check_loss(x, w, t, grad=TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cross_entropy_confident_and_hopeless(dtype):
    """Logits of hundreds: a probability of one for the target (loss and gradient next to nothing), or for another token."""
    x, w = normal((40, 64), TYPES[dtype], 1, 4.0), normal((300, 64), TYPES[dtype], 2, 4.0)
    best = (x.double() @ w.double().T).argmax(1).to(torch.int32)
    check_loss(x, w, best)
    check_loss(x, w, (best + 1) % 300)
    check_loss(x, w, best, scale=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cross_entropy_padding_hides_infinities(dtype):
    """Rows that do not count may hold anything; without one that counts everything is zero."""
    n, vocab, width = 100, 200, 72
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2)
    t = some_tokens(n, vocab, 3, padding=0.5)
    out = (t < 0) | (t >= vocab)
    clean = check_loss(x, w, t)
    x[out] = math.nan
    x[out.nonzero()[0, 0]] = math.inf
    c = B.make_cross_entropy(x, w, t)
    B.hbp_loss_cross_entropy(c)
    for name in ("loss", "row_loss", "dx", "dweight"):
        assert torch.equal(getattr(c, name), getattr(clean, name)), name
    assert bool((c.dx[out] == 0).all()) and bool((c.row_loss[out] == 0).all())
    none = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for mean in (True, False):
        c = B.make_cross_entropy(x, w, none, mean=mean)
        B.hbp_loss_cross_entropy(c)
        assert all(bool((v == 0).all()) for v in (c.loss, c.row_loss, c.dx, c.dweight))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cross_entropy_infinities_reach_their_row_only(dtype):
    x, w = normal((20, 64), TYPES[dtype], 1), normal((300, 64), TYPES[dtype], 2)
    t = some_tokens(20, 300, 3, padding=0.0)
    x[3, 5], x[4, 6] = math.nan, math.inf
    c = B.make_cross_entropy(x, w, t)
    B.hbp_loss_cross_entropy(c)
    rows = torch.arange(20, device="cuda")
    fine = (rows != 3) & (rows != 4)
    assert not bool(torch.isfinite(c.loss)[0]) and torch.equal(torch.isfinite(c.row_loss), fine)
    assert torch.equal(torch.isfinite(c.dx.float()).all(1), fine)


def test_cross_entropy_strides_what_is_not_wanted_and_nothing():
    big, wide = normal((50, 200), torch.bfloat16, 1), normal((90, 160), torch.bfloat16, 2)
    x, w, t = big[:, 8:136], wide[:, 16:144], some_tokens(50, 90, 3)
    room, grad = torch.full((60, 256), SENTINEL, dtype=torch.bfloat16, device="cuda"), torch.full((95, 144), SENTINEL, device="cuda")
    c = check_loss(x, w, t, dx=room[:50, 64:192], dweight=grad[:90, 8:136])
    assert bool((room[50:] == room[59, 0]).all()) and bool((room[:, :64] == room[59, 0]).all()) and bool((room[:, 192:] == room[59, 0]).all())
    assert bool((grad[90:] == SENTINEL).all()) and bool((grad[:, :8] == SENTINEL).all()) and bool((grad[:, 136:] == SENTINEL).all())
    for name in ("dx", "dweight"):
        d = B.make_cross_entropy(x, w, t)
        setattr(d, name, None)
        B.hbp_loss_cross_entropy(d)
        other = "dweight" if name == "dx" else "dx"
        assert torch.equal(getattr(d, other), getattr(c, other)) and torch.equal(d.loss, c.loss)
    d.row_loss = None
    d.loss.fill_(SENTINEL)
    B.hbp_loss_cross_entropy(d)
    assert torch.equal(d.loss, c.loss)
    one = x[:1].expand(50, 128)
    check_loss(one, w, t)
    e = B.make_cross_entropy(x[:0], w, t[:0])
    B.hbp_loss_cross_entropy(e)
    assert e.loss.item() == 0 and bool((e.dweight == 0).all())


# ---- together, streams, graphs --------------------------------------------------------------------------------------
def tied(seed, dtype=torch.bfloat16, n=200, vocab=700, width=128, counter=None):
    """A model of two ends that share a table: its embedding and its loss."""
    table = normal((vocab, width), dtype, seed, 0.1)
    tokens, targets = some_tokens(n, vocab, seed + 1), some_tokens(n, vocab, seed + 2)
    e = B.make_embedding(tokens, table, scale=3.0, dropout=B.make_dropout(0.2, 11, seed, counter))
    return e, B.make_cross_entropy(e.out, table, targets, dweight=e.dtable)


def step(e, c):
    B.hbp_embedding_forward(e)
    B.hbp_loss_cross_entropy(c)
    B.hbp_embedding_backward(e, c.dx, accumulate=True)


def results(e, c):
    return [v.clone() for v in (e.out, c.loss, c.row_loss, c.dx, e.dtable)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_both_ends_of_one_table(dtype):
    e, c = tied(1, TYPES[dtype])
    step(e, c)
    drop = (0.2, 11, 1)
    R.assert_within(e.out, *R.embedding(e.tokens, e.table, 3.0, drop), "out")
    want = R.cross_entropy(e.out, e.table, c.targets)
    R.assert_within(c.loss, *want["loss"], "loss")
    R.assert_within(c.dx, *want["dx"], "dx")
    more, bound = R.embedding_grad(e.tokens, c.dx, 700, 3.0, drop, torch.float32)
    R.assert_within(e.dtable, want["dweight"][0] + more, want["dweight"][1] + bound + 4 * R.F * (want["dweight"][0].abs() + more.abs()), "dtable")


def test_dropout_is_the_embeddings():
    """The mask on the way out of an embedding is hbp_dropout's."""
    e, _ = tied(2, torch.float32)
    B.hbp_embedding_forward(e)
    plain = B.make_embedding(e.tokens, e.table, scale=3.0, grad=False)
    B.hbp_embedding_forward(plain)
    out = torch.empty_like(plain.out)
    B.hbp_dropout(e.dropout, plain.out, out)
    assert torch.equal(out == 0, e.out == 0) and torch.allclose(out, e.out, rtol=4 * R.F, atol=0)


def test_another_stream_and_two_calls_at_once():
    a, b = tied(3), tied(4)
    want = []
    for m in (a, b):
        step(*m)
        want.append(results(*m))
        for v in (m[0].out, m[1].loss, m[1].row_loss, m[1].dx, m[0].dtable):
            v.fill_(SENTINEL)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for m, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                step(*m)
    torch.cuda.synchronize()
    assert same(results(*a), want[0]) and same(results(*b), want[1])


def test_captured_and_replayed():
    """A graph of a step, replayed between eager steps and with the counter moved on: every replay as the eager step of that counter."""
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    e, c = tied(5, counter=counter)
    want = []
    for i in range(3):
        counter.fill_(i)
        step(e, c)
        want.append(results(e, c))
    assert not torch.equal(want[0][0], want[1][0])
    counter.fill_(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(e, c)
    for i in (0, 1, 2, 1, 0):
        counter.fill_(i)
        for v in (e.out, c.loss, c.row_loss, c.dx, e.dtable):
            v.fill_(SENTINEL)
        c.workspace.fill_(255)
        e.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert same(results(e, c), want[i]), i
        step(e, c)
        assert same(results(e, c), want[i]), i


def test_around_a_stack():
    """Tokens to loss and back: embedding, a post-norm transformer stack of the library, the loss into the stack's e, exact
    backpropagation, the embedding's gradient; against 64-bit autograd of the whole."""
    import numpy as np
    from paper_2501_17086_amd import synth
    from tests.helpers import O, oracle_stack
    vocab, n, d = 300, 96, 64
    w = synth.scaled(synth.WORKLOADS["roberta_like"], name="ends", L=4, N=n, seq_len=32, d=d, heads=2, d_ff=128, dtype="f32", w1_std=0.0,
                     w2_std=0.0, w2_scale=0.6)
    inp = synth.make_inputs(w)
    p = B.allocate(w, inp)
    table = normal((vocab, d), torch.float32, 1)
    tokens, targets = some_tokens(n, vocab, 2), some_tokens(n, vocab, 3)
    e = B.make_embedding(tokens, table, out=p.x[0], dropout=B.make_dropout(0.1, 5))
    c = B.make_cross_entropy(p.x[-1], table, targets, dx=p.e, dweight=e.dtable)
    B.hbp_embedding_forward(e)
    B.hbp_forward(p)
    B.hbp_loss_cross_entropy(c)
    B.hbp_exact_backward(p)
    B.hbp_embedding_backward(e, p.g[0], accumulate=True)
    torch.cuda.synchronize()
    st = oracle_stack(w, inp)
    x0 = R.embedding(tokens, table, 1.0, (0.1, 5, 0))[0]
    sv = O.forward(st, x0.cpu().numpy())
    last = torch.from_numpy(np.asarray(sv["x"][-1])).cuda()
    loss = R.cross_entropy(last, table, targets)
    g = O.exact_backward(st, sv, loss["dx"][0].cpu().numpy())
    want = loss["dweight"][0] + R.embedding_grad(tokens, torch.from_numpy(np.asarray(g[0])).cuda(), vocab, 1.0, (0.1, 5, 0), torch.float32)[0]
    # (fp32: the stacks' tests allow 1e-5 in relative L2 of forward and gradients; here both come in)
    assert abs(c.loss.item() - loss["loss"][0].item()) < 2e-5 * loss["loss"][0].item()
    assert ((e.dtable.double() - want).norm() / want.norm()).item() < 2e-5
