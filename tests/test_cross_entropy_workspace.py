"""CPU-only: what the cross entropy asks for as its workspace."""
import ctypes as C

import pytest

from paper_2501_17086_amd import binding as B


def workspace(rows, vocab, width, dtype, gradients, grad_dtype=B.F32):
    n = C.c_size_t(0)
    desc = B.hbp_cross_entropy_desc(C.sizeof(B.hbp_cross_entropy_desc), dtype, grad_dtype, 1, 1.0, 1.0, rows, vocab, width)
    assert B.lib().hbp_cross_entropy_workspace_size(C.byref(desc), gradients, C.byref(n)) == 0, (rows, vocab, width, dtype, gradients)
    return n.value


@pytest.mark.parametrize("rows,vocab,width", [(65536, 512, 1024), (32768, 1000, 2048), (8192, 256, 65536), (16384, 16, 1024)])
def test_one_piece_keeps_dx_once_or_twice(rows, vocab, width):
    """Rows enough that no product of dx is shared out and the vocabulary is one piece: a product, and one for a rest of the vocabulary that is no
    whole slice; beside them dS and at most 16 shares of dweight."""
    more = workspace(rows, vocab, width, B.BF16, 1) - workspace(rows, vocab, width, B.BF16, 0)
    assert more <= 2 * rows * width * 4 + rows * vocab * 2 + 16 * vocab * width * 4 + 4096


@pytest.mark.parametrize("vocab", [1, 16, 31])
def test_a_vocabulary_below_a_slice_is_one_product(vocab):
    rows, width = 16384, 1024
    more = workspace(rows, vocab, width, B.BF16, 1) - workspace(rows, vocab, width, B.BF16, 0)
    assert more <= rows * width * 4 + rows * vocab * 2 + 16 * vocab * width * 4 + 4096


@pytest.mark.parametrize("rows,vocab,width", [(1825, 6000, 512), (3900, 8000, 512), (1, 50, 8), (8191, 100, 64)])
def test_fp32_rows_are_filled_up_to_eight(rows, vocab, width):
    """x's copy, five numbers a row, two for 64 of its logits, the logits; 256 bytes for each place to begin at."""
    n = (rows + 7) // 8 * 8
    assert workspace(rows, vocab, width, B.F32, 0) <= 4 * n * (width + 5 + 2 * ((vocab + 63) // 64) + vocab) + 10 * 256
