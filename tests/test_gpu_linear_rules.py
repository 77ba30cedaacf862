"""The layer's forward on both sides of every rule that chooses how few tokens are multiplied: tokens quantised by every
workgroup or in a launch of their own, four or sixteen wavefronts, few tokens or tiles, lengths around the steps of 64 and
batches of eight of them; against the definitions as in the other tests of the layer."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_linear_i8 import DEV, TYPES, check_sums, host, laid, quantized

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m, k, n", [
    (1, 1500, 5003),            # four wavefronts, each workgroup quantises
    (1, 8192, 4100), (1, 8193, 4100), (1, 8192, 4096), (1, 8193, 4096),     # what a workgroup holds, on both sides, four and sixteen
    (4, 1251, 8200), (4, 1667, 8200),                                       # so many workgroups a unit: not beyond 20,000 numbers
    (16, 512, 4097), (16, 513, 4096), (15, 37, 4099),
    (16, 4103, 4111), (17, 4103, 4111), (16, 2047, 100), (17, 2047, 100),   # the most tokens of one instruction
    (3, 63, 4097), (3, 64, 4097), (3, 65, 4097), (2, 2049, 17), (2, 511, 4500), (2, 2111, 4500), (16, 7, 4097), (16, 9, 33)])
def test_few_tokens_on_both_sides_of_the_rules(kind, m, k, n):
    rng = np.random.default_rng(m * 101 + k * 3 + n)
    x = laid((rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))).astype(np.float32), TYPES[kind], k + 3, 1)
    w = rng.integers(-127, 128, (n, k)).astype(np.int8)
    sw, bias = (np.exp(rng.standard_normal(n)) / 100).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    q, s = quantized(host(x), "rows")
    for ldw, offset in ((-(-k // 16) * 16, 0), (k, 1)):
        out = torch.full((m, n + 3), 7.0, dtype=TYPES[kind], device=DEV)
        rt.linear_i8(x, laid(w, torch.int8, ldw, offset), torch.as_tensor(sw, device=DEV), out[:, 1:n + 1],
                     bias=torch.as_tensor(bias, device=DEV))
        check_sums(out[:, 1:n + 1], kind, q, s, w, sw, bias)
        assert bool((out[:, 0] == 7).all()) and bool((out[:, n + 1:] == 7).all())


@pytest.mark.parametrize("rows, cols", [(64, 64 * 16), (64, 64 * 16 + 1), (33, 64 * 17), (64, 64 * 32 + 5), (5000, 17), (64, 64 * 513)])
@pytest.mark.parametrize("count", [1, 3, 17])
def test_narrow_matrices_on_both_sides_of_joining(rows, cols, count):
    """Up to sixteen blocks of 64 are added up by every workgroup, more by a launch; with many members fewer runs of more blocks."""
    if count * rows * cols > 4_000_000:
        count = 2
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows + cols + count)
    xs = [torch.randn(rows, cols, device=DEV, generator=gen) for _ in range(count)]
    outs = [torch.full_like(x, float("nan")) for x in xs]
    rt.orthogonalize(xs, outs)
    for x, out in zip(xs, outs):
        g = x.double() if rows <= cols else x.double().T.contiguous()
        g = g / (g.norm() + 1e-7)
        for a, b, c in [rt.QUINTIC] * 5:
            gram = g @ g.T.contiguous()
            g = a * g + (b * gram + c * gram @ gram) @ g
        want = g if rows <= cols else g.T
        # the room that the form in pairs of halves has for gradients
        assert float((out.double() - want).norm()) <= 2e-5 * float(want.norm())
