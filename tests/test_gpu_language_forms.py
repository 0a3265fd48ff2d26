"""Cross entropy at sizes whose rules take other paths than small ones do, element by element against the definitions in 64 bits."""
import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_gpu_language_ops import TYPES, check_loss, normal, results, same, some_tokens, step, tied

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 16, 31, 33])
def test_many_rows_against_a_handful(vocab, dtype):
    """dx fills the chip with a contraction shorter than a slice."""
    n, width = 16384, 256 if dtype == "f32" else 1024
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2, 0.05)
    check_loss(x, w, some_tokens(n, vocab, 3), grad=TYPES[dtype])


def test_long_contractions_are_shared_out():
    """fp32 sums of 2^20 equal terms: two entries, logits of zero, the factor 2, so that dS is 1 for the entry that is never the target and its dweight
    the plain sum of x = 4 / 3.  Added one by one each rounding may lean the same way: half a step of the sum so far, half the number of terms times
    f in all; in shares of 8192 and their join 4096 + 64 of them."""
    n = 1 << 20
    x, w = torch.full((n, 64), 4 / 3, device="cuda"), torch.zeros((2, 64), device="cuda")
    c = B.make_cross_entropy(x, w, torch.zeros(n, dtype=torch.int32, device="cuda"), mean=False, factor=2.0)
    B.hbp_loss_cross_entropy(c)
    want = torch.full((64,), n * x[0, 0].double().item(), dtype=torch.float64, device="cuda")
    R.assert_within(c.dweight[1], want, (4096 + 64) * R.F * want, "dweight")
    R.assert_within(c.dweight[0], -want, (4096 + 64) * R.F * want, "dweight of the target")


# (4100 against 22010: 85 x 4 tiles of dweight, of which a whole round of 256 goes alone; 22300: 87 x 4, which stay together; 16384 against 33100: two
# pieces whose weights are read from their copy, channels filled up to 288 and to 160)
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", [(4100, 22010, 1024), (4100, 22300, 1024), (16384, 33100, 264), (16384, 33100, 136)])
def test_many_tiles(n, vocab, width, grad):
    x, w = normal((n, width), torch.bfloat16, n), normal((vocab, width), torch.bfloat16, 2, 2.0 / width ** 0.5)
    check_loss(x, w, some_tokens(n, vocab, 3), grad=TYPES[grad])
    torch.cuda.empty_cache()


# sorted in blocks, and in more than 64 of them; logits in memory, and such that meet none: one piece, two, weights copied
MODELS = [(5000, 700, 128), (1000, 9300, 160), (70000, 9300, 160)]


@pytest.mark.parametrize("sizes", MODELS)
def test_two_steps_at_once(sizes):
    n, vocab, width = sizes
    a, b = (tied(s, n=n, vocab=vocab, width=width) for s in (3, 4))
    want = []
    for m in (a, b):
        step(*m)
        want.append(results(*m))
        for v in (m[0].out, m[1].loss, m[1].row_loss, m[1].dx, m[0].dtable):
            v.fill_(12345.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for m, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                step(*m)
    torch.cuda.synchronize()
    assert same(results(*a), want[0]) and same(results(*b), want[1])


@pytest.mark.parametrize("sizes", MODELS)
def test_captured_and_replayed(sizes):
    """Every replay as the eager step of its counter, with eager steps between the replays and nothing left over in the workspaces."""
    n, vocab, width = sizes
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    e, c = tied(5, n=n, vocab=vocab, width=width, counter=counter)
    want = []
    for i in range(2):
        counter.fill_(i)
        step(e, c)
        want.append(results(e, c))
    assert not torch.equal(want[0][0], want[1][0])
    counter.fill_(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(e, c)
    for i in (0, 1, 1, 0):
        counter.fill_(i)
        for v in (e.out, c.loss, c.row_loss, c.dx, e.dtable):
            v.fill_(12345.0)
        c.workspace.fill_(255)
        e.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert same(results(e, c), want[i]), i
        step(e, c)
        assert same(results(e, c), want[i]), i


@pytest.mark.parametrize("sizes", MODELS)
def test_both_ends_of_one_table(sizes):
    n, vocab, width = sizes
    e, c = tied(1, n=n, vocab=vocab, width=width)
    step(e, c)
    drop = (0.2, 11, 1)
    R.assert_within(e.out, *R.embedding(e.tokens, e.table, 3.0, drop), "out")
    want = R.cross_entropy(e.out, e.table, c.targets)
    for name in ("loss", "row_loss", "dx"):
        R.assert_within(getattr(c, name), *want[name], name)
    more, bound = R.embedding_grad(e.tokens, c.dx, vocab, 3.0, drop, torch.float32)
    R.assert_within(e.dtable, want["dweight"][0] + more, want["dweight"][1] + bound + 4 * R.F * (want["dweight"][0].abs() + more.abs()), "dtable")
    torch.cuda.empty_cache()
