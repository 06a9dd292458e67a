"""Sizes at the very end of what the operators on four-bit matrices take: refused before any launch, or not at all."""
import ctypes

import pytest

NULL, SHAPE, BF16 = 1, 2, 1
P = ctypes.c_void_p
BIG = 1 << 40      # addresses far apart, never followed


@pytest.fixture(scope="module")
def L():
    import paper_2308_14711_amd as F
    return F.lib()


def test_tiles_of_a_product_are_a_whole_number_for_each_xcd(L):
    """A launch ends before 2^24 blocks of 256 threads, and its blocks are a multiple of eight: 2^24 - 8 tiles are the most.  (A call that passes
    the checks of its sizes is refused for its missing pointer.)"""
    def product(tiles, a):
        assert tiles % 3 == 0
        return L.fff_mx4_product(None, P(a) if a else None, P(2 * BIG), P(3 * BIG), None, 2, P(4 * BIG), None, 128 * (tiles // 3), 32, 384, BF16, None, 0)
    most = (1 << 24) - 8
    for a in (0, 5 * BIG):
        assert product(most - most % 3, a) == NULL
        for tiles in range(most + 1, most + 9):
            if tiles % 3 == 0:
                assert product(tiles, a) == SHAPE, tiles

    def leaves(tiles):
        # pairs of one leaf: 64 a tile, and a part of a tile
        return L.fff_leaf_mx4_scratch_bytes(64 * (tiles - 1), 32, 32, 1, 1, 32) > 0
    assert leaves(most)
    for tiles in range(most + 1, most + 9):
        assert not leaves(tiles), tiles


def test_tiles_of_columns_to_quantise_end_at_a_launch(L):
    """2^24 tiles of 128 rows x 64 columns are one too many, whatever the tiles of a matrix."""
    def refused(batch, rows, cols):
        return L.fff_mx4_quantize(None, P(2 * BIG), P(3 * BIG), 1, None, batch, rows, cols, BF16) == SHAPE
    for rows, cols, tiles in ((1, 1, 1), (1, 129, 3), (300, 64, 3), (129, 200, 8), (640, 1, 5)):
        batch = ((1 << 24) - 1) // tiles
        assert not refused(batch, rows, cols) and refused(batch + 1, rows, cols), (rows, cols)
