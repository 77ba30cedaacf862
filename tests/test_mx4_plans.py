"""Which tiles the 4-bit products choose, on the host: that the sizes of the GPU tests reach all of them, and that no choice is a launch
that the device refuses."""
import pytest

import paper_2005_10761_amd as rt

from .test_gpu_mx4_tiles import PRODUCTS


def test_the_sizes_reach_every_tile():
    reached = {(p["edge"], p["runs"] > 1) for on_lines in (True, False) for p in (rt.product_mx4_plan(*s, on_lines) for s in PRODUCTS)}
    assert reached >= {(64, False), (64, True), (128, False), (128, True), (192, False), (256, False)}, reached


def test_refusals():
    for bad in ((0, 4, 4), (4, (1 << 22) + 1, 4), (4, 4, (1 << 22) + 1)):
        with pytest.raises(rt.RtopkError):
            rt.product_mx4_plan(*bad)


@pytest.mark.parametrize("m, n", [(1 << 22, 1 << 15), (1 << 15, 1 << 22), (1 << 22, 33_000), (1 << 22, 40_000), (1 << 22, 1 << 14)])
def test_a_launch_of_tiles_has_less_than_2_to_32_threads(m, n):
    """Results of up to 288 GB: a tile has 512 threads."""
    for k in (1, 8, 64, 100, 129, 500, 2000):
        for on_lines in (True, False):
            p = rt.product_mx4_plan(m, n, k, on_lines)
            assert p["tiles"] * p["runs"] * 512 < 1 << 32, (k, p)
