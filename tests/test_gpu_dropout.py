"""Dropout on the GPU: which elements are kept against Philox on the host, values within one rounding of each step."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests import four_bits as fb
from tests.test_gpu_mx4 import DEV, ROUND, TYPES, host, laid

pytestmark = pytest.mark.gpu


def check(out, kind, x, p, seed, step, residual=None):
    keep, factor = fb.kept(*x.shape, p, seed, step)
    more = 0.0 if residual is None else residual
    want = np.where(keep, np.where(keep, x, 0.0) * factor, 0.0) + more
    rel, least = ROUND[kind]
    # the factor's rounding, and one of the product and sum together
    room = 2.0 ** -24 * (np.abs(np.where(keep, x, 0.0) * factor) + np.abs(want) * 2)
    room = room + rel * (np.abs(want) + room) + least
    got = host(out)
    assert np.all(np.abs(got - want) <= room)
    dropped = ~keep
    assert np.array_equal(got[dropped], np.broadcast_to(more, x.shape)[dropped])


@pytest.mark.parametrize("kind, out_kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("rows, cols, pad, offset", [(1, 1, 0, 0), (1, 7, 0, 0), (1, 8, 0, 1), (3, 5, 0, 0), (3, 5, 2, 1), (700, 150, 0, 0),
                                                    (64, 96, 8, 0), (65, 40, 3, 1), (130, 1001, 1, 0), (1, 100_003, 0, 0), (2000, 3, 1, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_values(kind, out_kind, rows, cols, pad, offset, p):
    rng = np.random.default_rng(rows + cols)
    xd = laid(rng.standard_normal((rows, cols)), TYPES[kind], cols + pad, offset)
    resd = laid(rng.standard_normal((rows, cols)), TYPES[out_kind], cols + 2 * pad, offset)
    seed, step = 2 ** 40 + 17, 2 ** 33 + 1
    store = torch.full((rows * (cols + pad) + 3,), 9.0, dtype=TYPES[out_kind], device=DEV)
    out = store[1:1 + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    rt.dropout(xd, out, p, seed, step)
    check(out, out_kind, host(xd), p, seed, step)
    rt.dropout(xd, out, p, seed, step, residual=resd)
    check(out, out_kind, host(xd), p, seed, step, host(resd))
    beyond = store.clone()
    beyond[1:1 + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 9
    assert bool((beyond == 9).all())
    # the step from the device gives the same
    again = torch.empty(rows, cols, dtype=TYPES[out_kind], device=DEV)
    rt.dropout(xd, again, p, seed, torch.tensor([step], device=DEV), residual=resd)
    assert torch.equal(again, out)


def test_rows_that_lie_apart_draw_the_same():
    x = torch.randn(300, 77, device=DEV)
    apart = torch.empty(300, 90, device=DEV)[:, :77]
    apart.copy_(x)
    a, b = torch.empty_like(x), torch.empty(300, 80, device=DEV)[:, 3:]
    rt.dropout(x, a, 0.3, 1, 2)
    rt.dropout(apart, b, 0.3, 1, 2)
    assert torch.equal(a, b)
    flat = torch.empty(1, 300 * 77, device=DEV)
    rt.dropout(x.view(1, -1), flat, 0.3, 1, 2)
    assert torch.equal(flat.view_as(a), a)


def test_in_place_and_gradient():
    x, r = torch.randn(100, 130, device=DEV).to(torch.bfloat16), torch.randn(100, 130, device=DEV).to(torch.bfloat16)
    want = torch.empty_like(x)
    rt.dropout(x, want, 0.25, 3, 4, residual=r)
    for which in range(2):
        given = [x.clone(), r.clone()]
        rt.dropout(given[0], given[which], 0.25, 3, 4, residual=given[1])
        assert torch.equal(given[which], want)
    # out is linear in x, so a difference is the gradient's product with it: whole powers of two are exact
    ones, dx = torch.ones(100, 130, device=DEV), torch.empty(100, 130, device=DEV)
    rt.dropout(ones, dx, 0.5, 3, 4)
    a, b = torch.empty_like(dx), torch.empty_like(dx)
    rt.dropout(ones * 4, a, 0.5, 3, 4)
    rt.dropout(ones * 3, b, 0.5, 3, 4)
    assert torch.equal(a - b, dx) and set(dx.unique().tolist()) == {0.0, 2.0}


def test_what_is_dropped_counts_as_zero():
    x = torch.full((50, 64), float("nan"), device=DEV)
    x[:, ::2] = float("inf")
    out = torch.empty_like(x)
    rt.dropout(x, out, 0.5, 8, 9)
    keep, _ = fb.kept(50, 64, 0.5, 8, 9)
    got = host(out)
    assert np.array_equal(got == 0, ~keep) and np.isinf(got[:, ::2][keep[:, ::2]]).all() and np.isnan(got[:, 1::2][keep[:, 1::2]]).all()
    rt.dropout(x, out, 1.0, 8, 9)
    assert not out.any()


def test_share_of_what_is_kept():
    n = 1 << 20
    x = torch.ones(1, n, device=DEV)
    out = torch.empty_like(x)
    for p in (0.1, 0.5, 0.9):
        counts = []
        for seed, step in ((1, 1), (1, 2), (2, 1)):
            rt.dropout(x, out, p, seed, step)
            counts.append((out != 0).clone())
            # six deviations
            assert abs(float(counts[-1].double().mean()) - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17
        both = float((counts[0] & counts[1]).double().mean())
        assert abs(both - (1 - p) ** 2) < 6 * 0.5 / n ** 0.5


def test_places_beyond_32_bits():
    """The last elements of more than 2^32: their groups' upper halves."""
    rows, cols = (1 << 32) // 65_536 + 1, 65_536
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(x)
    rt.dropout(x, out, 0.5, 5, 6)
    base = (1 << 32) // 8
    want = fb.draws(base + np.arange(cols // 8), fb.FOR_DROPOUT, 5, 6).reshape(-1) >= 32_768
    assert np.array_equal(host(out[-1]) != 0, want)
    want = fb.draws(np.arange(cols // 8), fb.FOR_DROPOUT, 5, 6).reshape(-1) >= 32_768
    assert np.array_equal(host(out[0]) != 0, want)
