"""The matrix entry points on operands whose byte offsets pass 32 bits: what lies at both ends and around the places
where a shorter offset would wrap is compared with the definitions."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_linear_i8 import check_sums, host, quantized
from .test_gpu_orthogonal import SHARP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _around(count, *places):
    """Both ends of 0 .. count - 1 and the neighbours of `places`."""
    at = np.concatenate([np.arange(40), np.arange(count - 40, count)] + [np.arange(p - 20, p + 20) for p in places])
    return np.unique(at[(at >= 0) & (at < count)])


def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


@pytest.mark.parametrize("m", [2, 40])
def test_layer_of_more_than_four_gigabytes(m):
    k, n = 1901, 2_300_000                                  # odd rows: 4.4e9 bytes
    gen = _generator(m)
    w = torch.randint(-127, 128, (n, k), device=DEV, dtype=torch.int8, generator=gen)
    w_scale = torch.rand(n, device=DEV, generator=gen) + 0.5
    bias = torch.randn(n, device=DEV, generator=gen)
    x = torch.randn(m, k, device=DEV, generator=gen)
    out = torch.full((m, n), float("nan"), device=DEV)
    rt.linear_i8(x, w, w_scale, out, bias=bias)
    assert bool(torch.isfinite(out).all())
    q, s = quantized(host(x), "rows")
    at = _around(n, (1 << 31) // k, (1 << 32) // k, n // 2)
    pick = torch.as_tensor(at, device=DEV)
    check_sums(out[:, pick], "f32", q, s, host(w[pick]), host(w_scale[pick]), host(bias[pick]))


def test_output_of_more_than_four_gigabytes():
    m, n, k = 66_001, 66_003, 70                            # 4.4e9 numbers of two bytes
    gen = _generator(1)
    a = torch.randint(-127, 128, (m, 80), device=DEV, dtype=torch.int8, generator=gen)[:, :k]
    b = torch.randint(-127, 128, (n, 80), device=DEV, dtype=torch.int8, generator=gen)[:, :k]
    sa, sb = torch.rand(m, device=DEV, generator=gen) + 0.5, torch.rand(n, device=DEV, generator=gen) + 0.5
    out = torch.full((m, n), float("nan"), device=DEV, dtype=torch.bfloat16)
    rt.matmul_i8(a, sa, b, sb, out)
    rows = torch.as_tensor(_around(m, (1 << 31) // n, (1 << 30) // n, (1 << 32) // n), device=DEV)
    cols = torch.as_tensor(_around(n, n // 2), device=DEV)
    check_sums(out[rows][:, cols], "bf16", host(a[rows]), host(sa[rows]), host(b[cols]), host(sb[cols]))
    assert not bool(torch.isnan(out[rows]).any()) and not bool(torch.isnan(out[:, cols]).any())


def test_quantizing_more_than_eight_gigabytes():
    rows, cols = 2_097_157, 2101
    x = torch.randn(rows, cols, device=DEV, dtype=torch.bfloat16, generator=_generator(2))
    q, s = torch.full((rows, cols), 99, dtype=torch.int8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    rt.quantize_i8(x, q, s, along="rows")
    at = torch.as_tensor(_around(rows, (1 << 31) // cols, (1 << 30) // cols, (1 << 32) // cols), device=DEV)
    want_q, want_s = quantized(host(x[at]), "rows")
    assert np.array_equal(host(q[at]), want_q) and np.array_equal(host(s[at]), want_s)
    q, s = q.view(-1)[:rows * cols].view(cols, rows).fill_(99), torch.full((cols,), -1.0, device=DEV)
    rt.quantize_i8(x, q, s, along="columns")
    most = x.abs().amax(0).float()
    assert torch.equal(s, most / torch.full((), 127.0, device=DEV))
    for r0 in (0, (1 << 30) // cols - 30, (1 << 31) // cols - 30, rows - 60):
        want = torch.round(x[r0:r0 + 60].float() / s)       # (ties go to the even number, as in the definition)
        assert torch.equal(q[:, r0:r0 + 60].T, want.to(torch.int8))


def _turned(gram):
    """M with out = G M for tall G, from G^T G in binary64: five steps on it."""
    norm = gram.trace().sqrt() + 1e-7
    gram, total = gram / norm ** 2, torch.eye(gram.shape[0], dtype=torch.float64, device=DEV) / norm
    a, b, c = rt.QUINTIC
    for _ in range(5):
        step = a * torch.eye(gram.shape[0], dtype=torch.float64, device=DEV) + b * gram + c * gram @ gram
        gram, total = step @ gram @ step, total @ step
    return total


def _close(got, want, sharp):
    assert bool(torch.isfinite(got).all())
    assert float((got.double() - want).norm()) <= sharp * float(want.norm())


def test_orthogonalizing_a_long_matrix():
    rows, cols = 520, 1 << 21                               # 4.4e9 bytes, at the longest side
    x = torch.randn(rows, cols, device=DEV, generator=_generator(3))
    out = torch.full_like(x, float("nan"))
    rt.orthogonalize([x], [out])
    gram = torch.zeros(rows, rows, dtype=torch.float64, device=DEV)
    for part in x.split(1 << 18, dim=1):
        part = part.double()
        gram += part @ part.T.contiguous()
    turned = _turned(gram)
    for c0 in (0, cols // 2 - 500, cols - 1000):
        _close(out[:, c0:c0 + 1000], turned @ x[:, c0:c0 + 1000].double(), SHARP["pairs"])


def test_orthogonalizing_narrow_matrices_far_apart():
    rows, cols, count, pad = 1 << 21, 64, 3, 600            # rows 664 numbers apart: 5.6e9 bytes a matrix
    store = torch.randn(count, rows, cols + pad, device=DEV, generator=_generator(4))
    xs = [m[:, :cols] for m in store]
    outs = [torch.full((rows, cols), float("nan"), device=DEV) for _ in range(count)]
    rt.orthogonalize(xs, outs)
    for x, out in zip(xs, outs):
        turned = _turned(x.double().T.contiguous() @ x.double())
        for r0 in (0, rows // 2 - 500, (1 << 30) // (cols + pad) - 500, rows - 1000):
            _close(out[r0:r0 + 1000], x[r0:r0 + 1000].double() @ turned, SHARP["pairs"])
