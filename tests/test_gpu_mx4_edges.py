"""The 4-bit products at each tile, in one go and in runs of the contraction, with rows of no multiple of four and contractions of whole slices
(then the last slice's scales may not be loaded by fours), and of slices that end anywhere.
Which tile a size takes is checked on the host, beside the other plans."""
import pytest

from .test_gpu_mx4_tiles import test_products as check_product

pytestmark = pytest.mark.gpu

# (edge of the tiles, in runs): sizes m, n, k
BY_TILE = {
    (64, False): [(35, 39, 768), (97, 61, 1001)], (64, True): [(37, 43, 3328), (61, 35, 4999)],
    (128, False): [(262, 6941, 768)], (128, True): [(71, 3431, 11_776)],
    (192, False): [(2985, 2703, 768)], (192, True): [(134, 3495, 32_768)],
    (256, False): [(3001, 4501, 1024)], (256, True): [(387, 5463, 23_808), (425, 8856, 14_353)]}


@pytest.mark.parametrize("m, n, k", [size for sizes in BY_TILE.values() for size in sizes])
@pytest.mark.parametrize("aligned", [True, False])
def test_products_by_tile(m, n, k, aligned):
    check_product(m, n, k, aligned)
