"""Cross entropy of rows that are certain of their target, and of logits that are exact: what a row's loss and its target's coefficient
are then, in every form (logits and sums in one launch, logits in memory, logits that meet no memory)."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_gpu_language_ops import TYPES, normal

pytestmark = pytest.mark.gpu
SIZES = [(8, 2000, 256), (100, 30000, 264), (1000, 9300, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_certain_rows_have_no_negative_loss(n, vocab, width, dtype):
    """Rows that are their target's weights: its logit is 4 width, the others' next to 4 sqrt(width), their probabilities below e^-400 and so
    zero in 32 bits.  A loss is then never below zero, and a target's coefficient, all that its row of dweight holds, never above."""
    w = normal((vocab, width), TYPES[dtype], 1, 2.0)
    t = torch.randperm(vocab, generator=torch.Generator().manual_seed(2))[:n].int().cuda()
    x = w[t.long()].clone()
    c = B.make_cross_entropy(x, w, t, mean=False)
    B.hbp_loss_cross_entropy(c)
    s = x.double() @ w.double().T
    own = s.gather(1, t.long()[:, None])
    assert bool((own - s.scatter(1, t.long()[:, None], -math.inf).amax(1, keepdim=True) > 110).all())     # e^-110 is below fp32
    assert bool((c.row_loss >= 0).all()) and c.loss.item() >= 0
    R.assert_within(c.row_loss, torch.zeros(n, dtype=torch.float64, device="cuda"),
                    R.cross_entropy(x, w, t, mean=False)["row_loss"][1], "row_loss")
    along = (c.dweight[t.long()].double() * x.double()).sum(1) / x.double().square().sum(1)              # the coefficient
    assert bool((along <= 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES + [(100, 1 << 20, 64), (600, 20001, 1000), (1000, 9300, 160)])
def test_certain_rows_have_no_loss(n, vocab, width, dtype):
    """The same rows: a target's logit of 4 width cancels against the largest, bit by bit itself, and what is left is the logarithm of a sum of one
    term: three exponentials of a step each, two products and the logarithm, 12 f.  (A logit's own rounding is 2 width f and more.)  At 64 channels
    another of a million entries comes near: its term is known but for both logits' errors, (width + 3) f of the absolute terms' sum each."""
    w = normal((vocab, width), TYPES[dtype], 1, 2.0)
    t = torch.randperm(vocab, generator=torch.Generator().manual_seed(2))[:n].int().cuda()
    t[0] = vocab - 1
    t[1:][t[1:] == vocab - 1] = 0
    x = w[t.long()].clone()
    c = B.make_cross_entropy(x, w, t, mean=False)
    B.hbp_loss_cross_entropy(c)
    s = x.double() @ w.double().T
    s -= s.gather(1, t.long()[:, None])
    s.scatter_(1, t.long()[:, None], -math.inf)
    want = torch.log1p(s.exp().sum(1))
    bound = 12 * R.F + 2 * (width + 3) * R.F * x.double().square().sum(1) * want
    assert bool((c.row_loss >= 0).all())
    R.assert_within(c.row_loss, want, bound, "row_loss")
    along = (c.dweight[t.long()].double() * x.double()).sum(1) / x.double().square().sum(1)              # the coefficients
    once = torch.bincount(t.long(), minlength=vocab)[t.long()] == 1
    R.assert_within(along[once], torch.expm1(-want)[once], bound[once] + 2.0 ** -8 * want[once], "coefficients")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("n,vocab,width", SIZES + [(1024, 9216, 128)])
def test_losses_of_equal_exact_logits(n, vocab, width, scale, dtype):
    """Every logit is 21 * 5 = 105, exact in every order of its sum (one channel): exponentials of differences are ones, their sum the vocabulary's
    size, exact, and a row's loss its logarithm whatever the logits' size: the logarithm's rounding, 2 f at most, that of ln 2 and the product's, and
    another 2 f for the sums that a loss passes through."""
    x, w = torch.zeros((n, width), dtype=TYPES[dtype], device="cuda"), torch.zeros((vocab, width), dtype=TYPES[dtype], device="cuda")
    x[:, 5], w[:, 5] = 21.0, 5.0
    c = B.make_cross_entropy(x, w, torch.arange(n, dtype=torch.int32, device="cuda") % vocab, scale=scale, grad=False)
    B.hbp_loss_cross_entropy(c)
    want = torch.full((n,), math.log(vocab), dtype=torch.float64, device="cuda")
    R.assert_within(c.row_loss, want, 6 * R.F * want, "row_loss")
    R.assert_within(c.loss, want[:1], 7 * R.F * want[:1], "loss")
