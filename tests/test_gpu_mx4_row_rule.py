"""Quantisation along rows on both sides of the rule for the rows of a workgroup: 16-bit numbers always take one side, and the same numbers in
binary32 have to give the same bits on the other."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests import four_bits as fb

from .test_gpu_matrix_far import _generator
from .test_gpu_mx4 import host, room_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# 64 rows from two workgroups a unit on, of rows that are longer than there are rows; just below the first, and just below the second
@pytest.mark.parametrize("rows, cols", [(130, 100_003), (1, 262_145), (64, 261_633), (4000, 9001), (4160, 4161), (64, 261_632), (4160, 4160), (4161, 4160)])
def test_both_sides_give_the_same_bits(rows, cols):
    x = torch.randn(rows, cols, device=DEV, generator=_generator(rows + cols)).to(torch.bfloat16)
    x[0, 7], x[rows // 2, -1], x[rows - 1, cols // 2] = float("inf"), 3e38, float("nan")
    results = []
    for kind in (torch.bfloat16, torch.float32):
        q, s, (q_store, s_store) = room_for(rows, cols, 5, 3)
        rt.quantize_mx4(x.to(kind), q, s)
        results.append((q_store, s_store))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    q, s, _ = room_for(rows, cols)
    rt.quantize_mx4(x.float(), q, s)
    pick = sorted({0, rows // 2, rows - 1})
    want_q, want_s = fb.quantized(host(x[pick][:, -640 - cols % 32:]))
    some = -(-(640 + cols % 32) // 32)
    assert np.array_equal(host(s[-some:, pick]), want_s) and np.array_equal(host(q[pick][:, -want_q.shape[1] // 2:]), fb.packed(want_q))
