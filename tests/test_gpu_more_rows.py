"""The most rows and the most columns that the calls take, 2^22: quantisation, a layer, norm and dropout of narrow and of long matrices; and two
captured graphs, each with the workspace of its own capture, replayed in turn."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests import four_bits as fb

from .test_gpu_matrix_far import _around, _generator
from .test_gpu_mx4 import check, host, operand, room_for
from .test_gpu_norm import backward, forward, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = 1 << 22


@pytest.mark.parametrize("cols", [3, 40])
def test_most_rows(cols):
    gen = _generator(cols)
    x = torch.randn(MOST, cols, device=DEV, generator=gen)
    pick = torch.as_tensor(_around(MOST, MOST // 2), device=DEV)
    q, s, _ = room_for(MOST, cols)
    rt.quantize_mx4(x, q, s)
    want_q, want_s = fb.quantized(host(x[pick]))
    assert np.array_equal(host(q[pick]), fb.packed(want_q)) and np.array_equal(host(s[:, pick]), want_s)
    t, ts, _ = room_for(cols, MOST)
    rt.quantize_mx4(x, t, ts, along="columns")
    for first in (0, MOST // 2, MOST - 64):
        want_q, want_s = fb.quantized(host(x[first:first + 64]), "columns")
        assert np.array_equal(host(t[:, first // 2:first // 2 + 32]), fb.packed(want_q)) and np.array_equal(host(ts[first // 32:first // 32 + 2]), want_s)
    rng = np.random.default_rng(cols)
    wq, ws, w, w_scale = operand(rng, 33, cols, 120, 125)
    bias = torch.randn(33, device=DEV, generator=gen)
    y = torch.empty(MOST, 33, device=DEV)
    rt.linear_mx4(x, w, w_scale, y, bias=bias)
    check(y[pick], "f32", fb.values(*fb.quantized(host(x[pick]))), fb.values(wq, ws), host(bias))
    gamma, beta = torch.randn(cols, device=DEV, generator=gen), torch.randn(cols, device=DEV, generator=gen)
    h, mean, rstd = torch.empty_like(x), torch.empty(MOST, device=DEV), torch.empty(MOST, device=DEV)
    rt.layer_norm(x, gamma, beta, h, mean, rstd)
    (want, off), _, _ = forward(host(x[pick]), host(gamma), host(beta), 1e-5)
    within(h[pick], want, off, "y")
    dy, dx = torch.randn(MOST, cols, device=DEV, generator=gen), torch.empty_like(x)
    dgamma, dbeta = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    rt.layer_norm_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
    within(dx[pick], *backward(host(dy[pick]), host(x[pick]), host(mean[pick]), host(rstd[pick]), host(gamma), 0.0)[0], "dx")
    dh = dy.double() * (x.double() - mean[:, None].double()) * rstd[:, None].double()
    # runs of at most 2^13 rows a lane in binary32
    within(dgamma, host(dh.sum(0)), 2.0 ** -24 * (1 << 13) * host(dh.abs().sum(0)), "dgamma")
    within(dbeta, host(dy.double().sum(0)), 2.0 ** -24 * (1 << 13) * host(dy.double().abs().sum(0)), "dbeta")


@pytest.mark.parametrize("rows", [1, 3])
def test_most_columns(rows):
    gen = _generator(rows)
    x = torch.randn(rows, MOST, device=DEV, generator=gen)
    q, s, _ = room_for(rows, MOST)
    rt.quantize_mx4(x, q, s)
    want_q, want_s = fb.quantized(host(x[:, -640:]))
    assert np.array_equal(host(q[:, -320:]), fb.packed(want_q)) and np.array_equal(host(s[-20:]), want_s)
    t, ts, _ = room_for(MOST, rows)
    rt.quantize_mx4(x, t, ts, along="columns")
    want_q, want_s = fb.quantized(host(x[:, -640:]), "columns")
    assert np.array_equal(host(t[-640:]), fb.packed(want_q)) and np.array_equal(host(ts[:, -640:]), want_s)
    # a contraction of 2^22 numbers, and as many channels
    wq, ws, w, w_scale = operand(np.random.default_rng(rows), 5, MOST, 120, 125)
    y = torch.empty(rows, 5, device=DEV)
    rt.linear_mx4(x, w, w_scale, y)
    check(y, "f32", fb.values(fb.unpacked(host(q), MOST), host(s)), fb.values(wq, ws))
    short = torch.randn(rows, 40, device=DEV, generator=gen)
    wide, wide_scale = torch.randint(0, 256, (MOST, 20), device=DEV, dtype=torch.uint8, generator=gen), torch.full((2, MOST), 125, dtype=torch.uint8, device=DEV)
    out = torch.empty(rows, MOST, device=DEV)
    rt.linear_mx4(short, wide, wide_scale, out)
    check(out[:, -500:], "f32", fb.values(*fb.quantized(host(short))), fb.values(fb.unpacked(host(wide[-500:]), 40), host(wide_scale[:, -500:])))
    h, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    rt.layer_norm(x, None, None, h, mean, rstd)
    xd = host(x)
    within(mean, xd.mean(1), 2.0 ** -24 * np.abs(xd).mean(1) + 1e-12, "mean")
    within(rstd, 1 / np.sqrt(xd.var(1) + 1e-5), 8 * 2.0 ** -24 / np.sqrt(xd.var(1) + 1e-5), "rstd")
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(MOST, device=DEV), torch.empty(MOST, device=DEV)
    rt.layer_norm_backward(x, x, mean, rstd, None, dx, dgamma, dbeta)
    unit = (xd - host(mean)[:, None]) * host(rstd)[:, None]
    within(dgamma, (xd * unit).sum(0), 2.0 ** -24 * 16 * np.abs(xd * unit).sum(0), "dgamma")
    want = host(rstd)[:, None] * (xd - xd.mean(1, keepdims=True) - unit * (xd * unit).mean(1, keepdims=True))
    within(dx, want, 2.0 ** -24 * 64 * (np.abs(xd) + 1), "dx")


def test_two_graphs_in_turn():
    """Each capture takes its workspace from the memory of its own graph."""
    gen = _generator(9)
    m, k, n = 300, 900, 500
    runs = []
    for _ in range(2):
        x, dy = torch.randn(m, k, device=DEV, generator=gen), torch.randn(m, n, device=DEV, generator=gen)
        w = torch.randn(n, k, device=DEV, generator=gen)
        wq, ws, _ = room_for(n, k, 14, 12)
        wt, wts, _ = room_for(k, n, 6, 12)
        rt.quantize_mx4(w, wq, ws)
        rt.quantize_mx4(w, wt, wts, along="columns")
        y, dx, dw, db = torch.empty(m, n, device=DEV), torch.empty_like(x), torch.empty_like(w), torch.empty(n, device=DEV)

        def step(x=x, dy=dy, wq=wq, ws=ws, wt=wt, wts=wts, y=y, dx=dx, dw=dw, db=db):
            rt.linear_mx4(x, wq, ws, y)
            rt.linear_mx4_backward(dy, x, wt, wts, dx, dw, db, seed=1, step=2)

        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dw, db)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        runs.append((graph, (y, dx, dw, db), want, step))
    for turn in range(4):
        for graph, outs, want, step in runs:
            for t in outs:
                t.fill_(5)
        for graph, outs, want, step in runs if turn % 2 else runs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for graph, outs, want, step in runs:
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn
        runs[turn % 2][3]()
