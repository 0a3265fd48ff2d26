"""Cross entropy at sizes whose rules take other paths than small ones do, element by element against the definitions in 64 bits."""
import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_gpu_language_ops import TYPES, check_loss, normal, some_tokens

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
