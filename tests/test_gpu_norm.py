"""Layer norm and its gradients on the GPU against the formulas in binary64. The tolerances count what binary32 sums of a
row can round: a lane adds up to 32 numbers one after the other, then 7 steps over its wavefront and up to 16 over the
wavefronts: 64 roundings at most."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests.test_gpu_mx4 import DEV, ROUND, TYPES, host, laid

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                  # half a step of binary32, relative
SUM = 64 * U


def rounded(room, want, kind):
    rel, least = ROUND[kind]
    return room + rel * (np.abs(want) + room) + least


def within(got, want, room, what):
    got = host(got)
    assert got.shape == want.shape
    off = ~(np.abs(got - want) <= room)
    assert not off.any(), (what, int(off.sum()), np.argwhere(off)[:4], got[off][:4], want[off][:4], room[off][:4])


def forward(x, gamma, beta, eps):
    """(y, mean, rstd) and how far binary32 may be from each."""
    c = x.shape[1]
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    y = d * rstd * gamma + beta
    off_mean = (SUM + 2 * U) * np.abs(x).sum(1, keepdims=True) / c
    off_d = off_mean + U * np.abs(d)
    off_var = (2 * np.abs(d) * off_d + off_d ** 2).mean(1, keepdims=True) + (SUM + 4 * U) * (var + off_mean ** 2)
    off_rstd = 0.5 * off_var / (var + eps) * 1.2 + 4 * U
    off_y = np.abs(gamma) * rstd * (off_d + (np.abs(d) + off_d) * (off_rstd + 3 * U)) + 2 * U * np.abs(y) + U * np.abs(beta)
    return (y, off_y), (mean[:, 0], off_mean[:, 0]), (rstd[:, 0], (rstd * off_rstd)[:, 0])


def backward(dy, x, mean, rstd, gamma, add):
    """(dx, dgamma, dbeta) from the mean and rstd that are handed over, and how far binary32 may be from each."""
    rows, c = x.shape
    mean, rstd = mean[:, None], rstd[:, None]
    h, g = (x - mean) * rstd, dy * gamma
    m0, m1 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = rstd * (g - m0 - h * m1) + add
    off_m0 = (SUM + 3 * U) * np.abs(g).sum(1, keepdims=True) / c
    off_m1 = (SUM + 6 * U) * np.abs(g * h).sum(1, keepdims=True) / c
    off_dx = rstd * (U * np.abs(g) + off_m0 + np.abs(h) * off_m1 + 3 * U * np.abs(h * m1) + 4 * U * (np.abs(g) + np.abs(m0) + np.abs(h * m1)))
    off_dx = off_dx + 2 * U * (np.abs(dx) + np.abs(add))
    # sums over the rows, in any order
    off_gamma, off_beta = (rows + 8) * U * np.abs(dy * h).sum(0), (rows + 8) * U * np.abs(dy).sum(0)
    return (dx, off_dx), ((dy * h).sum(0), off_gamma), (dy.sum(0), off_beta)


SIZES = [(1, 1, 0, 0), (3, 2, 1, 1), (1, 1500, 0, 0), (5, 7, 0, 0), (4, 8, 3, 1), (1030, 40, 0, 0), (1100, 513, 2, 1), (1200, 1024, 0, 0),
         (33, 1025, 0, 0), (700, 1500, 0, 0), (9, 2047, 1, 0), (17, 4096, 8, 0), (6, 4099, 0, 0), (40, 8192, 0, 0), (5, 8200, 0, 0),
         (3, 16384, 0, 0), (4, 16385, 1, 1), (2, 50_001, 0, 0), (300, 96, 4, 2), (2500, 3, 0, 0), (5000, 260, 0, 0), (2048, 1024, 0, 0),
         (2049, 700, 1, 0), (1300, 2000, 0, 0), (600, 4000, 0, 0), (300, 8000, 0, 0), (150, 16_000, 0, 0), (130, 17_000, 0, 0)]


def rows_of(rng, rows, cols):
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))) + rng.standard_normal((rows, 1))
    if rows > 3:
        x[1] = 0.5                              # nothing varies: eps alone
        x[2] = 100 + rng.standard_normal(cols)  # a mean far from zero
    return x


@pytest.mark.parametrize("kind, out_kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows, cols, pad, offset", SIZES)
def test_forward_and_backward(kind, out_kind, rows, cols, pad, offset):
    rng = np.random.default_rng(rows * 31 + cols)
    xd = laid(rows_of(rng, rows, cols), TYPES[kind], cols + pad, offset)
    x = host(xd)
    gamma, beta = (1 + 0.2 * rng.standard_normal(cols)).astype(np.float32), rng.standard_normal(cols).astype(np.float32)
    gd, bd = torch.as_tensor(gamma, device=DEV), torch.as_tensor(beta, device=DEV)
    gamma, beta = gamma.astype(np.float64), beta.astype(np.float64)
    store = torch.full((rows, cols + 3), 9.0, dtype=TYPES[out_kind], device=DEV)
    out, mean, rstd = store[:, 1:1 + cols], torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    rt.layer_norm(xd, gd, bd, out, mean, rstd, eps=1e-5)
    (y, off_y), (m, off_m), (r, off_r) = forward(x, gamma, beta, 1e-5)
    within(mean, m, off_m, "mean")
    within(rstd, r, off_r, "rstd")
    within(out, y, rounded(off_y, y, out_kind), "y")
    assert bool((store[:, 0] == 9).all()) and bool((store[:, 1 + cols:] == 9).all())
    plain = torch.empty(rows, cols, dtype=TYPES[out_kind], device=DEV)
    rt.layer_norm(xd, None, None, plain)
    (y, off_y), _, _ = forward(x, 1.0, 0.0, 1e-5)
    within(plain, y, rounded(off_y, y, out_kind), "y without weights")
    dyd = laid(rng.standard_normal((rows, cols)) * 0.1, TYPES[out_kind], cols + 2 * pad, offset)
    addd = laid(rng.standard_normal((rows, cols)), TYPES[kind], cols + pad, 0)
    dx = torch.full((rows, cols + 1), 9.0, dtype=TYPES[kind], device=DEV)
    dgamma, dbeta = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dyd, xd, mean, rstd, gd, dx[:, :cols], dgamma, dbeta, add=addd)
    want = backward(host(dyd), x, host(mean), host(rstd), gamma, host(addd))
    within(dx[:, :cols], want[0][0], rounded(want[0][1], want[0][0], kind), "dx")
    within(dgamma, *want[1], "dgamma")
    within(dbeta, *want[2], "dbeta")
    assert bool((dx[:, cols] == 9).all())
    # each alone, and without weight and addition
    alone = torch.empty(rows, cols, dtype=TYPES[kind], device=DEV)
    rt.layer_norm_backward(dyd, xd, mean, rstd, None, alone)
    want = backward(host(dyd), x, host(mean), host(rstd), 1.0, 0.0)
    within(alone, want[0][0], rounded(want[0][1], want[0][0], kind), "dx alone")
    only = torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dyd, xd, mean, rstd, gd, None, only)
    within(only, *want[1], "dgamma alone")
    rt.layer_norm_backward(dyd, xd, mean, rstd, gd, None, None, only)
    within(only, *want[2], "dbeta alone")
    # the same bits every time
    again = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dyd, xd, mean, rstd, gd, dx[:, :cols], *again, add=addd)
    assert torch.equal(again[0], dgamma) and torch.equal(again[1], dbeta)


@pytest.mark.parametrize("rows, cols", [(7, 5), (50, 1500), (1500, 200), (4, 20_000), (3000, 1000), (2500, 3000), (130, 17_000)])
def test_in_place(rows, cols):
    rng = np.random.default_rng(rows)
    x = torch.as_tensor(rows_of(rng, rows, cols), device=DEV).to(torch.bfloat16)
    gamma, beta = torch.randn(cols, device=DEV), torch.randn(cols, device=DEV)
    mean, rstd, want = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(x)
    rt.layer_norm(x, gamma, beta, want, mean, rstd)
    got = x.clone()
    rt.layer_norm(got, gamma, beta, got)
    assert torch.equal(got, want)
    dy, add = torch.randn_like(x), torch.randn_like(x)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta, add=add)
    for which in range(3):
        given = [dy.clone(), x.clone(), add.clone()]
        sums = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        rt.layer_norm_backward(given[0], given[1], mean, rstd, gamma, given[which], *sums, add=given[2])
        assert torch.equal(given[which], dx) and torch.equal(sums[0], dgamma) and torch.equal(sums[1], dbeta), which


def test_rows_that_are_not_numbers_stay_by_themselves():
    x = torch.randn(6, 300, device=DEV)
    clean = torch.empty_like(x)
    rt.layer_norm(x, None, None, clean)
    x[1, 7], x[3, 299], x[4, 0] = float("nan"), float("inf"), float("-inf")
    y = torch.empty_like(x)
    rt.layer_norm(x, None, None, y)
    assert bool(y[[1, 3, 4]].isnan().all()) and torch.equal(y[[0, 2, 5]], clean[[0, 2, 5]])


def test_large_and_small_numbers():
    rng = np.random.default_rng(1)
    for scale in (1e-20, 1e-3, 1e15):
        x = (rng.standard_normal((8, 1000)) * scale).astype(np.float32)
        out = torch.empty(8, 1000, device=DEV)
        rt.layer_norm(torch.as_tensor(x, device=DEV), None, None, out, eps=0.0 if scale > 1e-19 else 1e-5)
        (y, off), _, _ = forward(x.astype(np.float64), 1.0, 0.0, 0.0 if scale > 1e-19 else 1e-5)
        within(out, y, off + 1e-44, scale)


def test_no_rows():
    x = torch.empty(0, 40, device=DEV)
    none = torch.empty(0, device=DEV)
    rt.layer_norm(x, None, None, torch.empty_like(x))
    dgamma, dbeta = torch.full((40,), 3.0, device=DEV), torch.full((40,), 3.0, device=DEV)
    rt.layer_norm_backward(x, x, none, none, None, torch.empty_like(x), dgamma, dbeta)
    assert not dgamma.any() and not dbeta.any()


def test_gradients_against_differences():
    """The whole chain in binary32 against central differences of the loss in binary64 from the formula."""
    rng = np.random.default_rng(2)
    rows, cols = 5, 37
    x, dy = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    gamma, beta = rng.standard_normal(cols), rng.standard_normal(cols)
    x, dy, gamma, beta = (v.astype(np.float32) for v in (x, dy, gamma, beta))
    to = lambda v: torch.as_tensor(v, device=DEV)   # noqa: E731
    y, mean, rstd = torch.empty(rows, cols, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    rt.layer_norm(to(x), to(gamma), to(beta), y, mean, rstd)
    dx, dgamma, dbeta = torch.empty(rows, cols, device=DEV), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(to(dy), to(x), mean, rstd, to(gamma), dx, dgamma, dbeta)
    loss = lambda x, g, b: (forward(x, g, b, 1e-5)[0][0] * dy.astype(np.float64)).sum()   # noqa: E731
    given = [v.astype(np.float64) for v in (x, gamma, beta)]
    h = 1e-5
    for which, got in enumerate((dx, dgamma, dbeta)):
        want = np.empty(given[which].shape)
        for at in np.ndindex(want.shape):
            sides = []
            for sign in (1, -1):
                moved = [v.copy() for v in given]
                moved[which][at] += sign * h
                sides.append(loss(*moved))
            want[at] = (sides[0] - sides[1]) / (2 * h)
        # differences: h^2 and 2^-52 / h of the loss's terms, 1e-9 together; binary32: 64 roundings of terms of a few units
        assert np.abs(host(got) - want).max() < 64 * 8 * U * np.abs(want).max() + 1e-8
