"""Layer norm of rows whose mean is far larger than what varies around it. The mean that a row's sum gives is off by the sum's
roundings, `first` below; what is left over is a sum of the small differences from it, so that results are off by
roundings of the differences, and by nothing at all where all numbers of a row are equal."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests.test_gpu_mx4 import DEV, TYPES, host
from tests.test_gpu_norm import SUM, U, rounded, within

pytestmark = pytest.mark.gpu
# a width for each way to hold a row, odd ones among them; beyond 16384 rows are summed in binary64
WIDTHS = [3, 40, 1000, 1024, 1500, 2048, 3001, 4096, 8192, 12_001, 16_384, 20_000, 50_001]
EPS = float(np.float32(1e-5))


def weights(cols):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(cols)
    return torch.randn(cols, device=DEV, generator=gen), torch.randn(cols, device=DEV, generator=gen)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_equal_numbers_give_beta(kind, cols):
    """d is exact (mean is within 36 roundings of x: 15 of a lane's sum, 20 of lanes' and wavefronts', the division), and a multiple j <= 72 of
    x's last place; cols j < 2^24, so the sum of all d, its division by cols and d less it are exact too."""
    values = [0.1, -0.7, 3.3, 11000.1] + ([100000.3, -1.2345e7, 1.1e30, 1.7e-30] if kind != "f16" else [])
    column = torch.tensor(values, dtype=torch.float32, device=DEV).to(TYPES[kind])
    x = column[:, None].repeat(1, cols)
    gamma, beta = weights(cols)
    out, mean, rstd = torch.empty(len(values), cols, device=DEV), torch.empty(len(values), device=DEV), torch.empty(len(values), device=DEV)
    rt.layer_norm(x, gamma, beta, out, mean, rstd)
    assert torch.equal(mean, column.float())
    assert torch.equal(out, beta.expand_as(out))
    assert np.abs(host(rstd) * np.sqrt(EPS) - 1).max() <= 4 * U
    rt.layer_norm(x, gamma, beta, out, eps=0.0)
    assert bool(out.isnan().all())


def forward(x, gamma, beta):
    """(y, mean, rstd) and how far they may be off."""
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + EPS)
    first = (SUM + 2 * U) * np.abs(x).mean(1, keepdims=True)            # of the first mean
    left = (SUM + 3 * U) * (np.abs(d).mean(1, keepdims=True) + first)   # of what is left over
    off_d = U * (np.abs(d) + first) + left + U * np.abs(d)
    off_var = (SUM + 6 * U) * (var + first ** 2) + 2 * first * left + left ** 2
    off_rstd = 0.5 * off_var / (var + EPS) * 1.2 + 4 * U                # relative
    y = d * rstd * gamma + beta
    off_y = np.abs(gamma) * rstd * (off_d + (np.abs(d) + off_d) * (off_rstd + 3 * U)) + 2 * U * np.abs(y) + U * np.abs(beta)
    return (y, off_y), (mean[:, 0], (left + U * np.abs(mean))[:, 0]), (rstd[:, 0], (rstd * off_rstd)[:, 0])


@pytest.mark.parametrize("kind, out_kind", [("f32", "f32"), ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("cols", WIDTHS)
def test_means_far_from_zero(kind, out_kind, cols):
    rng = np.random.default_rng(cols)
    far = {"f32": [1e3, 1e4, -1e6, 3e7], "bf16": [100.0, -3e4], "f16": [100.0, -3e4]}[kind]
    spread = [1.0 if kind == "f32" else abs(c) / 50 for c in far]
    rows = [c + s * rng.standard_normal(cols) for c, s in zip(far, spread)]
    # one number far from all others, at either end; one last place between two halves of a row
    lone = rng.standard_normal((2, cols))
    lone[0, 0] = lone[1, -1] = 1e4
    two = np.full(cols, 11000.1 if kind == "f32" else 1000.0)
    two[::2] *= 1 + 2.0 ** (-23 if kind == "f32" else -7)
    xd = torch.as_tensor(np.stack(rows + [lone[0], lone[1], two]).astype(np.float32), device=DEV).to(TYPES[kind])
    x = host(xd)
    gamma, beta = weights(cols)
    n = len(x)
    out, mean, rstd = torch.empty(n, cols, dtype=TYPES[out_kind], device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    rt.layer_norm(xd, gamma, beta, out, mean, rstd)
    (y, off_y), (m, off_m), (r, off_r) = forward(x, host(gamma), host(beta))
    within(mean, m, off_m, "mean")
    within(rstd, r, off_r, "rstd")
    within(out, y, rounded(off_y, y, out_kind), "y")


@pytest.mark.parametrize("cols", [700, 1500, 5000, 9000, 16_384, 20_000])
def test_means_near_zero_are_off_by_roundings_of_their_sum(cols):
    """Not by those of the differences from them: these are rounded the same way within a power of two, so that their sum is off by
    parts of their number, not of its root."""
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((200, cols)).astype(np.float32)
    mean = torch.empty(200, device=DEV)
    rt.layer_norm(torch.as_tensor(x, device=DEV), None, None, torch.empty(200, cols, device=DEV), mean)
    # a partial sum of j numbers is sqrt(j) large, its rounding U / sqrt(3) of that; squares of all roundings: a lane's up to 16 numbers give 8 cols,
    # 6 steps over lanes 6 cols, up to 16 wavefronts 8 cols: sqrt(22 / 3 cols) U of the sum, and one U of the mean, 1 / sqrt(cols) large, for the
    # division; 3.7 in all, here twice that
    off = host(mean) - x.astype(np.float64).mean(1)
    assert np.sqrt((off ** 2).mean()) <= 7.5 * U / np.sqrt(cols)
