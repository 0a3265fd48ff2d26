"""CPU-only: what the cross entropy asks for as its workspace."""
import ctypes as C
import math
import random

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


def sizes(seed, count):
    """Sizes over the whole range, many of them at a tile's, a slice's or a piece's border."""
    rng = random.Random(seed)

    def near(lo, hi):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        if rng.random() < 0.5:
            unit = rng.choice((32, 64, 256))
            v = round(v / unit) * unit + rng.choice((-32, -8, -1, 0, 0, 0, 1, 8, 31, 32))
        return max(1, min(hi, int(v)))
    for _ in range(count):
        rows, vocab = near(1, rng.choice((4096, 1 << 20))), near(1, rng.choice((1 << 17, 1 << 17, 1 << 24)))
        width = near(8, rng.choice((2048, 65536))) // 8 * 8
        if rng.random() < 0.3:
            width = (width + 255) // 256 * 256
        yield rows, vocab, min(65536, max(8, width)), rng.choice((B.F32, B.BF16, B.BF16))


def test_every_product_has_its_room():
    """The library goes through a call's products as its launches do and refuses sizes of which one lacks room in what `carve` reserves: there are
    none such."""
    for size in sizes(1, 60000):
        assert workspace(*size, 1) > workspace(*size, 0) > 0, size


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_sizes_around_a_tile(dtype):
    for rows in (1, 8, 255, 256, 257, 4095, 4096, 8192, 16384, 1 << 20):
        for tiles in (0, 1, 85, 86, 87, 141, 142, 255, 256, 257, 512):
            for rest in (0, 1, 31, 32, 33, 255):
                for width in (8, 128, 256, 264, 512, 1000, 1024, 2048):
                    vocab = 256 * tiles + rest
                    if vocab:
                        assert workspace(rows, vocab, width, dtype, 1) > workspace(rows, vocab, width, dtype, 0) > 0


def test_fp32_contractions_are_shared_out_by_8192():
    """Room for a share of each 8192 of a product's contraction: the vocabulary for dx, the rows for dweight."""
    vocab, rows, width = 1 << 20, 1 << 20, 64
    assert workspace(8, vocab, width, B.F32, 1) - workspace(8, vocab, width, B.F32, 0) >= vocab // 8192 * 8 * width * 4
    assert workspace(rows, 2, width, B.F32, 1) - workspace(rows, 2, width, B.F32, 0) >= rows // 8192 * 2 * width * 4 + rows * width * 4
