"""Which tiles and forms of steps the matrix calls choose, on the host: that the sizes of the GPU tests reach all of them, and that
no choice is a launch that the device refuses."""
import pytest

import paper_2005_10761_amd as rt

from .test_gpu_matrix_tiles import MATRICES, PRODUCTS


def test_the_sizes_reach_every_tile():
    reached = {(p["edge"], p["runs"] > 1) for on_lines in (True, False) for p in (rt.product_plan(*s[2:], on_lines) for s in PRODUCTS)}
    assert reached >= {(e, r) for e in (128, 192, 256) for r in (True, False)}
    grams, squares, nexts, twos = set(), set(), set(), set()
    for products in ("pairs", "halves"):
        for count, rows, cols in MATRICES:
            p = rt.orthogonalize_plan(count, rows, cols, products)
            assert not p["narrow"]
            grams.add((products, p["gram_edge"], p["joined"]))
            squares.add((products, p["square_edge"]))
            nexts.add((products, p["next_edge"], rows > cols))
            twos.add((products, p["two_at_a_time"], rows > cols))
    edges, both = (64, 128, 192, 256), ("pairs", "halves")
    assert grams >= {(p, e, j) for p in both for e in edges for j in (0, 1)} - {("halves", 256, 1)}     # (no size was found that takes it)
    assert squares == {(p, e) for p in both for e in edges}
    assert nexts == {(p, e, o) for p in both for e in edges for o in (False, True)}
    assert twos == {("pairs", t, o) for t in (0, 1) for o in (False, True)} | {("halves", 0, o) for o in (False, True)}


def test_refusals():
    for bad in ((0, 4, 4), (4, (1 << 22) + 1, 4), (4, 4, (1 << 22) + 1)):
        with pytest.raises(rt.RtopkError):
            rt.product_plan(*bad)
    for bad in (dict(count=0), dict(count=17), dict(rows=0), dict(cols=(1 << 21) + 1), dict(coefficients=(9.0, 0.0, 0.0))):
        with pytest.raises(rt.RtopkError):
            rt.orthogonalize_plan(**{**dict(count=1, rows=100, cols=200), **bad})
    assert rt.orthogonalize_plan(2, 64, 5000)["narrow"] == 1


@pytest.mark.parametrize("m, n", [(1 << 22, 1 << 15), (1 << 15, 1 << 22), (1 << 22, 33_000), (1 << 22, 40_000), (1 << 22, 1 << 14)])
def test_a_launch_of_tiles_has_less_than_2_to_32_threads(m, n):
    """Results of up to 288 GB: a tile has 512 threads."""
    for k in (1, 8, 64, 100, 129, 500):
        for on_lines in (True, False):
            p = rt.product_plan(m, n, k, on_lines)
            assert p["tiles"] * p["runs"] * 512 < 1 << 32, (k, p)
