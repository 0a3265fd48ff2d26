"""Cross entropy against weights that hold infinities and NaNs: entries of the vocabulary masked by a weight of -inf, and batches in which no
row, or not every row, counts.  Sizes of all three forms: logits and sums in one launch, logits in memory, logits that meet no memory
(bf16; whole tiles, and tiles with a rest)."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_gpu_language_ops import SENTINEL, TYPES, normal, some_tokens

pytestmark = pytest.mark.gpu
SIZES = [(8, 2000, 64), (100, 30000, 264), (1024, 9216, 128), (1000, 9300, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES)
@pytest.mark.parametrize("value", [-math.inf, math.inf, math.nan])
def test_no_row_counts(n, vocab, width, dtype, value):
    """Zeros everywhere, whatever the weights hold."""
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2)
    w[5], w[vocab - 1, 3], w[vocab // 2, 7] = value, value, value
    c = B.make_cross_entropy(x, w, torch.full((n,), -1, dtype=torch.int32, device="cuda"))
    for v in (c.loss, c.row_loss, c.dx, c.dweight):
        v.fill_(SENTINEL)
    B.hbp_loss_cross_entropy(c)
    for name in ("loss", "row_loss", "dx", "dweight"):
        assert bool((getattr(c, name) == 0).all()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES)
@pytest.mark.parametrize("padding", [0.0, 0.3])
def test_entries_masked_by_a_weight(n, vocab, width, dtype, padding):
    """A channel that is positive in every row, and a weight of -inf on it: the entry's probability is zero.  Everything is as without the
    entry (sums are of zeros more), its own dweight zero; dx's channel is 0 times -inf and not looked at."""
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2, 2.0 / math.sqrt(width))
    x[:, 3] = x[:, 3].abs() + 0.5
    masked = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    masked[torch.tensor([0, 17, 130, vocab // 2, vocab - 2], device="cuda")] = True
    w[masked, 3] = -math.inf
    left = (~masked).nonzero()[:, 0]
    t = some_tokens(n, left.numel(), 3, padding=padding)               # among the entries that are left
    on = (t >= 0) & (t < left.numel())
    targets = torch.where(on, left[t.long().clamp(0, left.numel() - 1)], torch.full_like(left[:1], -1)).int()
    c = B.make_cross_entropy(x, w, targets)
    B.hbp_loss_cross_entropy(c)
    want = R.cross_entropy(x, w[left].contiguous(), t)
    for name in ("loss", "row_loss"):
        R.assert_within(getattr(c, name), *want[name], name)
    others = torch.arange(width, device="cuda") != 3
    R.assert_within(c.dx[:, others], *(v[:, others] for v in want["dx"]), "dx")
    assert bool((c.dx[~on] == 0).all())
    R.assert_within(c.dweight[left], *want["dweight"], "dweight")
    assert bool((c.dweight[masked] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES)
@pytest.mark.parametrize("padding", [0.0, 0.3])
def test_entries_masked_by_the_lowest_value(n, vocab, width, dtype, padding):
    """The same with the type's lowest value, whole blocks of 128 entries among the masked: logits from -1.7e38 to -infinity, finite ones beyond the largest
    number once they are taken to base 2.  Zero times such a weight is zero: dx too is as without the entries."""
    x, w = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2, 2.0 / math.sqrt(width))
    x[:, 3] = x[:, 3].abs() + 0.5
    masked = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    masked[120:520] = True
    masked[vocab - 3:] = True
    w[masked, 3] = torch.finfo(TYPES[dtype]).min
    left = (~masked).nonzero()[:, 0]
    t = some_tokens(n, left.numel(), 3, padding=padding)
    on = (t >= 0) & (t < left.numel())
    targets = torch.where(on, left[t.long().clamp(0, left.numel() - 1)], torch.full_like(left[:1], -1)).int()
    c = B.make_cross_entropy(x, w, targets)
    B.hbp_loss_cross_entropy(c)
    want = R.cross_entropy(x, w[left].contiguous(), t)
    for name in ("loss", "row_loss", "dx"):
        R.assert_within(getattr(c, name), *want[name], name)
    R.assert_within(c.dweight[left], *want["dweight"], "dweight")
    assert bool((c.dweight[masked] == 0).all())
