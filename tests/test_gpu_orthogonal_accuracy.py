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


@pytest.mark.parametrize("products", ["pairs", "halves"])
@pytest.mark.parametrize("rows, cols, count", [(40, 300, 2), (300, 64, 1), (64, 1300, 1), (100, 130, 3), (300, 90, 1), (520, 4610, 1)])
def test_norms_far_below_eps(rows, cols, count, products):
    """Below eps every step multiplies the matrix by a, and by 2^-22 (2^-11) more or less: D is stored relative to the
    h that it is around, and moves the polynomial by (|b| + 2 |c|) h <= 2.6 a of that, the polynomial and X by one more each. Five
    steps leave 23 roundings: 5.5e-6 with pairs, 1.1e-2 with halves if all of them had one sign, a third of that otherwise. Members of
    a batch have norms of their own."""
    rng = np.random.default_rng(rows + cols)
    limit = {"pairs": 2e-5, "halves": 2.0 ** -8}[products]
    for ratio, eps in ((1.0, 2.0), (0.2, 1.0), (1e-2, 1e-3), (1e-4, 1e-7), (1e-6, 1.0), (1e-8, 1e-7), (1e-14, 1.0), (1e-7, 1e-7), (1e-22, 1e5)):
        gs = []
        for i in range(count):
            g = rng.standard_normal((rows, cols))
            gs.append((g / np.sqrt((g * g).sum()) * ratio * eps * 30.0 ** i).astype(np.float32))
        xs = [torch.as_tensor(g, device=DEV) for g in gs]
        outs = [torch.full((rows, cols), float("nan"), device=DEV) for _ in gs]
        rt.orthogonalize(xs, outs, eps=eps, products=products)
        for g, out in zip(gs, outs):
            want, _ = reference(g, eps=float(np.float32(eps)), products=products)
            assert relative(host(out), want) <= limit, (ratio, eps)


def test_steps_that_shrink_keep_their_bits():
    """Polynomials far below one: what is stored is scaled by what the coefficients can leave."""
    rng = np.random.default_rng(1)
    for rows, cols in ((50, 400), (90, 200), (200, 90)):
        g = rng.standard_normal((rows, cols)).astype(np.float32)
        for steps in ([(1e-3, 0.0, 0.0)] * 4, [(0.01, 0.005, 0.0)] * 3 + [(2.0, -1.0, 0.1)]):
            x, out = torch.as_tensor(g, device=DEV), torch.empty(rows, cols, device=DEV)
            rt.orthogonalize([x], [out], coefficients=steps)
            assert relative(host(out), reference(g, steps)[0]) <= 2e-5, steps
