"""The most rows that the 8-bit calls take, 2^22, at the lengths whose rows have a workgroup of 1024 threads each: more threads
than a launch has along one dimension."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt

from .test_gpu_linear_i8 import check_sums, host, quantized

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = 1 << 22


@pytest.mark.parametrize("rows, cols, kind", [(ROWS, 8201, torch.bfloat16), (ROWS - 1, 500, torch.bfloat16), (ROWS, 1030, torch.float16),
                                              ((1 << 20) + 1, 16_390, torch.float16)])
def test_most_rows(rows, cols, kind):
    if torch.cuda.mem_get_info()[1] < 150 << 30:
        pytest.skip("needs 140 GB of device memory")
    gen = torch.Generator(device=DEV)
    gen.manual_seed(cols)
    x = torch.empty(rows, cols, device=DEV, dtype=kind)
    for part in x.split(1 << 20):                           # (pieces: what it takes besides x stays small)
        part.normal_(generator=gen)
    at = torch.as_tensor(np.unique(np.concatenate([np.arange(20), np.arange(rows - 20, rows), np.arange((1 << 20) - 10, min((1 << 20) + 10, rows)),
                                                   np.arange(rows // 2 - 10, rows // 2 + 10)])), device=DEV)
    want_q, want_s = quantized(host(x[at]), "rows")
    q, s = torch.full((rows, cols), 99, dtype=torch.int8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    rt.quantize_i8(x, q, s)
    assert np.array_equal(host(q[at]), want_q) and np.array_equal(host(s[at]), want_s)
    assert bool((s > 0).all())
    del q
    # and through a layer, whose workspace holds as many
    w = torch.randint(-127, 128, (3, cols), device=DEV, dtype=torch.int8, generator=gen)
    w_scale = torch.rand(3, device=DEV, generator=gen) + 0.5
    out = torch.full((rows, 3), float("nan"), device=DEV)
    rt.linear_i8(x, w, w_scale, out)
    assert bool(torch.isfinite(out).all())
    check_sums(out[at], "f32", want_q, want_s, host(w), host(w_scale))
    del x, out
    torch.cuda.empty_cache()
