"""That the sizes of the products by tile take the tile that they stand for, however their rows lie, and that every tile is among them."""
import pytest

import paper_2005_10761_amd as rt

from .test_gpu_mx4_edges import BY_TILE


def test_every_tile_in_one_go_and_in_runs():
    assert set(BY_TILE) == {(edge, runs) for edge in (64, 128, 192, 256) for runs in (False, True)}


@pytest.mark.parametrize("tile", list(BY_TILE))
def test_a_size_takes_its_tile(tile):
    for size in BY_TILE[tile]:
        for on_lines in (True, False):
            p = rt.product_mx4_plan(*size, on_lines)
            assert (p["edge"], p["runs"] > 1) == tile, (size, p)
    m, n, k = BY_TILE[tile][0]
    assert (m % 4 or n % 4) and k % 256 == 0 and k >= 3 * 256
