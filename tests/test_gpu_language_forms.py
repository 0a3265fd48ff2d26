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
