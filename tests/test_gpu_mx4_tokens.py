"""A token through a layer in 4 bits alone and among others, up to the 16 that a call of few tokens takes: the same sums in the same order."""
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_matrix_far import _generator
from .test_gpu_mx4_tiles import _operand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# on both sides of the rules for the wavefronts and for quantising in the product's launch
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k, n", [(512, 64), (513, 64), (1500, 2049), (4096, 300), (200, 4097), (5000, 4100), (33, 2000)])
def test_a_token_has_the_same_bits_alone_and_among_others(kind, k, n):
    gen = _generator(k + n)
    w, w_scale = _operand(n, k, gen, True, 118, 122)
    x = torch.randn(16, k, device=DEV, generator=gen).to(kind)
    bias = torch.randn(n, device=DEV, generator=gen)
    among, alone = torch.empty(16, n, device=DEV), torch.empty(1, n, device=DEV)
    for count in (2, 5, 16):
        rt.linear_mx4(x[:count], w, w_scale, among[:count], bias=bias)
        for token in {0, count // 2, count - 1}:
            rt.linear_mx4(x[token:token + 1], w, w_scale, alone, bias=bias)
            assert torch.equal(alone[0], among[token]), (count, token)
