"""Norm, 4-bit product, dropout onto the residual path, and back, as a training program calls them: eagerly, captured into
one graph whose step number advances on the device, and on two streams at once; the weights' gradients go on to the encoder."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests import four_bits as fb
from tests.test_gpu_mx4 import DEV, host

pytestmark = pytest.mark.gpu


class Block:
    """x + dropout(norm(x) w^T + b), and its gradients."""

    def __init__(self, tokens, width, seed, p=0.1):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device=DEV)   # noqa: E731
        f32 = torch.float32
        self.m, self.k, self.seed, self.p = tokens, width, seed, p
        self.w = torch.randn(width, width, device=DEV, generator=gen) / width ** 0.5
        self.gamma, self.beta, self.bias = (torch.randn(width, device=DEV, generator=gen) for _ in range(3))
        self.x = torch.randn(tokens, width, device=DEV, generator=gen).to(torch.bfloat16)
        self.dout = (0.01 * torch.randn(tokens, width, device=DEV, generator=gen)).to(torch.bfloat16)
        store = -(-width // 32) * 16
        self.wq, self.wt = new(width, store, dtype=torch.uint8)[:, :(width + 1) // 2], new(width, store, dtype=torch.uint8)[:, :(width + 1) // 2]
        self.ws, self.wts = (new(-(-width // 32), -(-width // 16) * 16, dtype=torch.uint8)[:, :width] for _ in range(2))
        self.h, self.y, self.out, self.dy, self.dh, self.dx = (new(tokens, width) for _ in range(6))
        self.mean, self.rstd = new(tokens, dtype=f32), new(tokens, dtype=f32)
        self.dw, self.db = new(width, width, dtype=f32), new(width, dtype=f32)
        self.dgamma, self.dbeta = new(width, dtype=f32), new(width, dtype=f32)

    def step(self, step, stream=None):
        at = {"stream": stream}
        rt.quantize_mx4(self.w, self.wq, self.ws, **at)
        rt.quantize_mx4(self.w, self.wt, self.wts, along="columns", **at)
        rt.layer_norm(self.x, self.gamma, self.beta, self.h, self.mean, self.rstd, **at)
        rt.linear_mx4(self.h, self.wq, self.ws, self.y, bias=self.bias, **at)
        rt.dropout(self.y, self.out, self.p, self.seed, step, residual=self.x, **at)
        rt.dropout(self.dout, self.dy, self.p, self.seed, step, **at)
        rt.linear_mx4_backward(self.dy, self.h, self.wt, self.wts, self.dh, self.dw, self.db, seed=self.seed, step=step, **at)
        rt.layer_norm_backward(self.dh, self.x, self.mean, self.rstd, self.gamma, self.dx, self.dgamma, self.dbeta, add=self.dout, **at)

    def results(self):
        return [t.clone() for t in (self.h, self.y, self.out, self.dy, self.dh, self.dx, self.dw, self.db, self.dgamma, self.dbeta)]


@pytest.mark.parametrize("tokens, width", [(70, 150), (512, 256), (1, 64), (16, 1500)])
def test_a_step_against_the_formulas(tokens, width):
    b = Block(tokens, width, 3)
    b.step(11)
    # from what each call was given: the calls' own tests hold their results, this one how they go together
    x, h = host(b.x), host(b.h)
    normal = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + 1e-5)
    assert np.abs(h - (normal * host(b.gamma) + host(b.beta))).max() <= 2.0 ** -8 * np.abs(h).max() * 1.01
    y = fb.values(*fb.quantized(h)) @ fb.values(*fb.quantized(host(b.w))).T + host(b.bias)
    assert np.abs(host(b.y) - y).max() <= 2.0 ** -8 * np.abs(y).max() * 1.01
    keep, factor = fb.kept(tokens, width, b.p, 3, 11)
    assert np.abs(host(b.out) - (keep * factor * host(b.y) + x)).max() <= 2.0 ** -8 * np.abs(host(b.out)).max() * 1.01
    assert np.abs(host(b.dy) - keep * factor * host(b.dout)).max() <= 2.0 ** -8 * np.abs(host(b.dy)).max() * 1.01
    dw = fb.values(*fb.quantized(host(b.dy), "columns", 3, 11)) @ fb.values(*fb.quantized(h, "columns")).T
    assert np.abs(host(b.dw) - dw).max() <= 1e-5 * np.abs(dw).max()
    dh = fb.values(*fb.quantized(host(b.dy), "rows", 3, 11)) @ fb.values(*fb.quantized(host(b.w), "columns")).T
    assert np.abs(host(b.dh) - dh).max() <= 2.0 ** -8 * np.abs(dh).max() * 1.01
    g = host(b.dh) * host(b.gamma)
    dx = (g - g.mean(1, keepdims=True) - normal * (g * normal).mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + 1e-5) + host(b.dout)
    assert np.abs(host(b.dx) - dx).max() <= (2.0 ** -8 + 1e-4) * np.abs(dx).max()
    # the gradients are what the encoder takes
    for grad in (b.dw.reshape(-1), b.dgamma):
        d = grad.numel()
        k, r = max(1, d // 50), max(1, d // 10)
        idx, val = torch.empty(k, dtype=torch.int32, device=DEV), torch.empty(k, device=DEV)
        ws = torch.empty(rt.encode_workspace_bytes(d, r, k), dtype=torch.uint8, device=DEV)
        rt.encode(grad, torch.zeros_like(grad), r, k, 3, 11, idx, val, ws)
        assert torch.equal(val, grad[idx.long()])


def test_a_replayed_graph_draws_anew():
    b = Block(130, 96, 5, p=0.3)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    b.step(step)                                    # (everything is loaded and sized before the capture)
    want = []
    for i in range(4):
        b.step(100 + i)
        want.append(b.results())
    assert not torch.equal(want[0][2], want[1][2]) and not torch.equal(want[0][6], want[1][6])
    step.fill_(99)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step.add_(1)
        b.step(step)
    step.fill_(99)
    other = Block(64, 64, 6)
    for i in range(4):
        for t in (b.h, b.y, b.out, b.dy, b.dh, b.dx, b.dw, b.db, b.dgamma, b.dbeta):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(b.results(), want[i])), i
        other.step(i)                               # eager work in between


def test_two_streams_at_once():
    blocks = [Block(300, 256, 8), Block(200, 320, 9)]
    want = []
    for b in blocks:
        b.step(1)
        want.append(b.results())
        b.step(2)
    streams = [torch.cuda.Stream() for _ in blocks]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, s in zip(blocks, streams):
            b.step(1, stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(g, v) for g, v in zip(b.results(), w))


def test_calls_on_the_current_stream():
    b = Block(100, 128, 4)
    b.step(1)
    want = b.results()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.x.mul_(0.5)
        b.x.mul_(2.0)
        b.step(1)
    stream.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(b.results(), want))
