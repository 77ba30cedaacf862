"""How near orthogonalised matrices are to the iteration in binary64 where roundings matter most: one direction much stronger
than the others, and norms far below eps."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_orthogonal import DEV, TYPES, host, reference

pytestmark = pytest.mark.gpu


def relative(got, want):
    return np.sqrt(((got - want) ** 2).sum()) / np.sqrt((want ** 2).sum())


@pytest.mark.parametrize("rows, cols", [(256, 1400), (1400, 256), (60, 1100)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("strength", [30, 100, 1000])
def test_a_strong_direction_does_not_cost_the_weak_ones_their_bits(strength, kind, rows, cols):
    """Noise, and one direction `strength` times as large in every element: a number stored with the unit u is off by u times
    the strong direction's element there, `strength` u of the noise's, and all weak directions grow alike. So with pairs (u = 2^-22)
    four roundings that matter leave 4 strength 2^-22; and a bfloat16 result is rounded by 2^-9 at most. Halves would
    lose 2048 times as much, so they are for callers who ask for them."""
    rng = np.random.default_rng(strength + rows)
    g = rng.standard_normal((rows, cols)) + strength * np.outer(rng.standard_normal(rows), rng.standard_normal(cols))
    x = torch.as_tensor(g, device=DEV).to(TYPES[kind])
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    rt.orthogonalize([x], [out])
    want, _ = reference(host(x))
    assert relative(host(out), want) <= 2.0 ** -9 + 4 * strength * 2.0 ** -22
