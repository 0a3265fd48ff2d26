"""What bf16 gradients of the cross entropy lose to their roundings, in relative L2: narrower than bounds that add up every rounding's half step, so that
what keeps two of them out, the rest of a target's coefficient in dx and the power of two in place of the factor, is seen to work.  A rounding's mean
square is a twelfth of its step's, and a step 2^-7 of a value at most: 2^-7 / sqrt(12) = 0.00226."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_gpu_language_ops import normal

pytestmark = pytest.mark.gpu
ONE = 2.0 ** -7 / math.sqrt(12)
# one launch for logits and sums; logits in memory; logits that meet no memory.  1 / rows is 1.0039 times a power of two: half a step beside 1
SIZES = [(255, 2000, 256), (255, 30000, 128), (1020, 9300, 128)]


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_dx_keeps_its_targets_coefficient(n, vocab, width):
    """Targets of a probability of 0.498047, whose coefficient, 0.501953, lies half a step from its neighbours, 0.0039 of it; it carries most of dx, as the
    other half of the mass is spread over the vocabulary.  Allowed is dx's own rounding, and a tenth for that of the others, whose
    probabilities' squares add up to next to nothing."""
    w = normal((vocab, width), torch.bfloat16, 1, 1.0 / math.sqrt(width))
    t = torch.randperm(vocab, generator=torch.Generator().manual_seed(2))[:n].int().cuda()
    wd, along = w.double(), w[t.long()].double()
    lo, hi = torch.zeros((n, 1), dtype=torch.float64, device="cuda"), torch.full((n, 1), 100.0, dtype=torch.float64, device="cuda")
    for _ in range(60):                                    # how long x has to be
        mid = (lo + hi) / 2
        p = torch.softmax(mid * along @ wd.T, 1).gather(1, t.long()[:, None])
        lo, hi = torch.where(p < 0.498047, mid, lo), torch.where(p < 0.498047, hi, mid)
    x = (mid * along).bfloat16()
    c = B.make_cross_entropy(x, w, t)
    B.hbp_loss_cross_entropy(c)
    assert off(c.dx, R.cross_entropy(x, w, t)["dx"][0]) < 1.1 * ONE


@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_dweight_keeps_its_factor(n, vocab, width):
    """Mean over 255 (1020) rows, each probability about 1 / vocabulary: the targets' coefficients are the factor but for that much, and its rounding to
    bf16, 0.0039, would be all of their rows' error.  Rows of dweight with targets, fp32; allowed are twice the two roundings of a coefficient:
    1 - 1 / vocabulary is next to 1 (off by 1 / vocabulary), and that of the other rows' probabilities, next to nothing."""
    x, w = normal((n, width), torch.bfloat16, 1, 0.05), normal((vocab, width), torch.bfloat16, 2, 0.05)
    t = (torch.arange(n, device="cuda") % 50).int()
    c = B.make_cross_entropy(x, w, t)
    B.hbp_loss_cross_entropy(c)
    assert off(c.dweight[:50], R.cross_entropy(x, w, t)["dweight"][0][:50]) < 2 / vocab + 1e-4


@pytest.mark.parametrize("n,vocab,width", SIZES)
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_gradients_of_plain_rows(n, vocab, width, grad):
    """One rounding for dS and one for the result where it is bf16."""
    x, w = normal((n, width), torch.bfloat16, 1), normal((vocab, width), torch.bfloat16, 2, 2.0 / math.sqrt(width))
    t = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(3)).int().cuda()
    c = B.make_cross_entropy(x, w, t, dweight=torch.empty((vocab, width), dtype=grad, device="cuda"))
    B.hbp_loss_cross_entropy(c)
    want = R.cross_entropy(x, w, t, grad_dtype=grad)
    assert off(c.dweight, want["dweight"][0]) < ONE * (math.sqrt(2) if grad == torch.bfloat16 else 1)
    assert off(c.dx, want["dx"][0]) < ONE * math.sqrt(2)
    assert off(c.loss, want["loss"][0]) < 16 * R.F and off(c.row_loss, want["row_loss"][0]) < 16 * R.F


@pytest.mark.parametrize("n,vocab,width", [(1, 50, 64), (1, 131072, 1024), (2, 300, 128), (5, 70, 2048), (8, 16384, 256), (64, 5000, 256), (128, 700, 1032),
                                           (120, 30000, 264), (3, (1 << 20) + 300, 8)])
def test_gradients_of_few_rows(n, vocab, width):
    """A row of dweight is a sum of few coefficients, whose roundings do not average out: dS keeps two terms here, each rounding half a step, 2^-8 of what
    the one before left out, 2^-16 together.  Beside it the logits' own errors in a coefficient, (width + 3) f of their size at most and a fraction
    of it on the average: as much again."""
    x, w = normal((n, width), torch.bfloat16, 1), normal((vocab, width), torch.bfloat16, 2, 1.0 / math.sqrt(width))
    t = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(3)).int().cuda()
    want = R.cross_entropy(x, w, t)
    for grad in (torch.float32, torch.bfloat16):
        c = B.make_cross_entropy(x, w, t, dweight=torch.empty((vocab, width), dtype=grad, device="cuda"))
        B.hbp_loss_cross_entropy(c)
        assert off(c.dweight, want["dweight"][0]) < (2.0 ** -15 if grad == torch.float32 else 1.1 * ONE)
        assert off(c.dx, want["dx"][0]) < 1.1 * ONE
