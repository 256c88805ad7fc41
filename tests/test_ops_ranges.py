"""Sizes and positions past 32 bits are refused, not cut to their low half (no GPU: nothing is enqueued)."""
import pytest

from paper_2607_12287_amd import incvit

T = 1 << 34   # an address that is never read
ROPE = incvit.make_rope(64, (8, 12, 12))


@pytest.mark.parametrize("grid", [(1, 2, 2, 2 ** 31), (1, 2, 2, 0, -2 ** 31 - 1), (1, 2, 2, 0, 0, 2 ** 32 + 7), (2 ** 32 + 1, 2, 2),
                                  (1, 2 ** 32 + 2, 2), (1, 2, -2 ** 32 + 2)])
def test_grids_past_32_bits(grid):
    with pytest.raises(ValueError):
        incvit.incvit_rope_table_grids(ROPE, [(1, 2, 2), grid], 1, T)
    with pytest.raises(ValueError):
        incvit.rope_table(ROPE, grids=[(1, 2, 2), grid], device="cuda:0")


@pytest.mark.parametrize("merge", [2 ** 32 + 1, 2 ** 31, -2 ** 32 + 1])
def test_merge_past_32_bits(merge):
    with pytest.raises(ValueError):
        incvit.incvit_rope_table_grids(ROPE, [(1, 2, 2)], merge, T)
    with pytest.raises(ValueError):
        incvit.rope_table(ROPE, grids=[(1, 2, 2)], merge=merge, device="cuda:0")


@pytest.mark.parametrize("pairs", [(-2 ** 32 + 16, 16), (0, 16), (2 ** 32 + 16, -2 ** 32, 8)])
def test_pairs_past_32_bits(pairs):
    with pytest.raises(ValueError):
        incvit.make_rope(64, pairs)


def test_the_ends_of_32_bits_are_taken():
    assert incvit.incvit_rope_table_grids(ROPE, [(1, 2, 2, 2 ** 31 - 1, -2 ** 31, 5)], 2 ** 31 - 1, T) == incvit.INCVIT_ERR_SHAPE
    assert incvit.incvit_rope_table_grids(ROPE, [], 1, T) == incvit.INCVIT_OK


def test_most_rows_of_the_8_bit_products():
    most = 2 ** 31 - 65
    assert incvit.incvit_qlinear_rows_bytes(most, 64) == (most + 15) // 16 * (1024 + 64)
    assert incvit.incvit_qlinear_rows_bytes(most + 1, 64) == 0
    assert incvit.incvit_qlinear_quantize_rows(1, most + 1, 64, T, 64, 0, 0, 1e-6, 2 * T) == incvit.INCVIT_ERR_ARG
