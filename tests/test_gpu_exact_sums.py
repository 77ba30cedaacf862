"""Sums over the most rows and the longest contractions, of numbers that make them exact: products are multiples of 1/4 or 1/2, and partial
sums in any order stay far below 2^22. Results are compared bit for bit, so that a run, a workgroup or a row that is left out shows."""
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_matrix_far import _generator
from .test_gpu_mx4 import room_for
from .test_gpu_mx4_tiles import LEVELS, _numbers, _operand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = 1 << 22


def _levels(rows, cols, gen, dtype=torch.bfloat16):
    """Numbers that 4 bits have, with a 6 or -6 in each block of 32 along both: all scales are 1."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEV).to(dtype)
    out = torch.empty(rows, cols, dtype=dtype, device=DEV)
    for at in range(0, rows, 1 << 19):
        out[at:at + (1 << 19)] = table[torch.randint(0, 16, out[at:at + (1 << 19)].shape, device=DEV, generator=gen)]
    for lines in (out[::32], out[:, ::32]):
        lines.copy_(torch.randint(0, 2, lines.shape, device=DEV, generator=gen) * 12 - 6)
    return out


def _product(a, b):
    """a^T b in binary64, a part of the rows at a time."""
    total = torch.zeros(a.size(1), b.size(1), dtype=torch.float64, device=DEV)
    for at in range(0, a.size(0), 1 << 19):
        total += a[at:at + (1 << 19)].double().T @ b[at:at + (1 << 19)].double()
    return total


@pytest.mark.parametrize("k, n", [(40, 40), (3, 64), (64, 1), (70, 33)])
def test_a_layers_backward_of_the_most_tokens(k, n):
    gen = _generator(k + n)
    dy, x, w = _levels(MOST, n, gen), _levels(MOST, k, gen), _levels(n, k, gen, torch.float32)
    turned, turned_scale, _ = room_for(k, n)
    rt.quantize_mx4(w, turned, turned_scale, along="columns")
    dx, dw, db = torch.empty_like(x), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    rt.linear_mx4_backward(dy, x, turned, turned_scale, dx, dw, db)
    want = _product(dy, x)
    # products are multiples of 1/4, a row's and a column's sum far below 2^22
    assert 0 < float(want.abs().max()) < 2.0 ** 21
    assert torch.equal(dw, want.float())
    assert torch.equal(db, dy.double().sum(0).float()) and bool(db.any())
    for at in (0, MOST // 2, MOST - 4096):
        assert torch.equal(dx[at:at + 4096], (dy[at:at + 4096].double() @ w.double()).float().to(dx.dtype))
    alone = torch.empty_like(x)
    rt.linear_mx4_backward(dy, None, turned, turned_scale, alone, None)
    assert torch.equal(alone, dx)


@pytest.mark.parametrize("m", [1, 3, 16, 17, 90])
def test_the_longest_contraction(m):
    gen = _generator(m)
    x = _levels(m, MOST, gen)
    w, w_scale = _operand(5, MOST, gen, True)
    want = _product(x.T, _numbers(w, w_scale, MOST).T.contiguous())
    assert 0 < float(want.abs().min()) and float(want.abs().max()) < 2.0 ** 21
    out = torch.empty(m, 5, device=DEV)
    rt.linear_mx4(x, w, w_scale, out)
    assert torch.equal(out, want.float())
    q, s, _ = room_for(m, MOST)
    rt.quantize_mx4(x, q, s)
    turned = torch.empty(5, m, device=DEV)
    rt.matmul_mx4(w, w_scale, q, s, turned)
    assert torch.equal(turned, want.float().T)


# one of each way to hold a row, and beyond; 512 workgroups keep their sums where a row is held, 128 runs of rows where not
@pytest.mark.parametrize("rows, cols", [(MOST, 3), (MOST, 40), (300_001, 1000), (200_003, 1500), (60_001, 4096), (30_001, 8192), (9000, 16_000), (5000, 17_001)])
def test_norm_sums_over_many_rows(rows, cols):
    gen = _generator(rows + cols)
    whole = lambda: torch.randint(-2, 3, (rows, cols), device=DEV, generator=gen, dtype=torch.int8).to(torch.bfloat16)   # noqa: E731
    x, dy = whole(), whole()
    mean = torch.randint(-1, 2, (rows,), device=DEV, generator=gen).float()
    rstd = torch.exp2(torch.randint(-1, 2, (rows,), device=DEV, generator=gen).float())
    # terms are multiples of 1/2 of at most 12
    want, plain = torch.zeros(cols, dtype=torch.float64, device=DEV), torch.zeros(cols, dtype=torch.float64, device=DEV)
    largest = torch.zeros(cols, dtype=torch.float64, device=DEV)
    for at in range(0, rows, 1 << 15):
        some = slice(at, min(rows, at + (1 << 15)))
        terms = dy[some].double() * (x[some].double() - mean[some, None].double()) * rstd[some, None].double()
        want, plain = want + terms.sum(0), plain + dy[some].double().sum(0)
        largest = torch.maximum(largest, want.abs())
    assert float(largest.max()) < 2.0 ** 22 and bool(want.any()) and bool(plain.any())
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dy, x, mean, rstd, None, dx, dgamma, dbeta)
    assert torch.equal(dgamma, want.float()) and torch.equal(dbeta, plain.float())
    # without dx: by runs of rows
    rt.layer_norm_backward(dy, x, mean, rstd, None, None, dgamma.fill_(7), dbeta.fill_(7))
    assert torch.equal(dgamma, want.float()) and torch.equal(dbeta, plain.float())
