"""The host definitions that the GPU tests of 4-bit numbers and draws compare with, pinned by hand and by Philox's
known answers."""
import os

import numpy as np

from tests import four_bits as fb


def test_philox_known_answers():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")
    seen = 0
    for line in open(path):
        words = line.split("#")[0].split()
        if len(words) < 10:
            continue
        numbers = [int(w, 16) for w in words[-10:]]
        got = fb.philox(np.array([numbers[:4]], np.uint64), numbers[4:6])
        assert [int(v) for v in got[0]] == numbers[6:]
        seen += 1
    assert seen >= 3


def test_draws_are_the_words_halves():
    words = fb.philox(np.array([[5, 2 << 24 | 1, 7, 9]], np.uint64), (11, 13))[0]
    got = fb.draws([5 + (1 << 32)], 2, 11 + (13 << 32), 7 + (9 << 32))[0]
    assert [int(v) for v in got] == [int(w) >> s & 0xFFFF for w in words for s in (0, 16)]


def test_nearest_numbers_by_hand():
    row = np.zeros((1, 40))
    row[0, :12] = [6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 6.99, -0.0]
    row[0, 32:36] = [7, 3.49, 3.5, 0.5]         # 7 would round to 8: the block's scale is 2
    q, scale = fb.quantized(row)
    assert scale.shape == (2, 1) and list(scale[:, 0]) == [127, 128]
    assert [float(fb.VALUES[n]) for n in q[0, :11]] == [6, -6, 0, 1, 1, 2, 2, 4, 4, -4, 6] and q[0, 11] == 8
    assert list(fb.values(q, scale)[0, 32:36]) == [8, 3, 4, 0]
    assert list(fb.unpacked(fb.packed(q), 40)[0]) == list(q[0])


def test_scales_at_the_ends():
    x = np.zeros((5, 32))
    x[1, 0], x[2, 0], x[3, 0], x[4, 0] = 2.0 ** -149, 3.4028234663852886e38, np.nan, np.inf
    q, scale = fb.quantized(x)
    assert list(scale[0]) == [0, 0, 253, 255, 255] and not q[3:].any() and q[2, 0] == 6


def test_drawn_numbers_keep_the_mean():
    x = np.full((1, 32), 0.0)
    x[0] = np.linspace(-6, 6, 32)
    total = sum(fb.values(*fb.quantized(x, seed=3, step=s)) for s in range(4000)) / 4000
    # a step is 2 at most, so a mean's deviation is at most 1 / sqrt(4000): six of them
    assert np.abs(total - x).max() < 6 / np.sqrt(4000)
    q, scale = fb.quantized(x, seed=3, step=0)
    assert scale[0, 0] == 127 and np.array_equal(fb.values(q, scale)[0, [0, 31]], [-6, 6])
