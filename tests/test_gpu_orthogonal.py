"""Orthogonalised updates on the GPU against the iteration in binary64.

The tolerance follows the roundings. Let u be the unit roundoff of the numbers between the products (2^-22 for pairs of
halves, 2^-11 for halves). In a step from X, with f = |X|_F and h >= its largest singular value, the stored A is off by
(u + K 2^-24) f^2 at most (K terms in binary32), which moves the new X by (|b| h + 2 |c| h^3) times that; the stored B
is off by (u + 2 K 2^-24) (|b| + |c| h^2) f^2 (A's Frobenius norm is at most h f, so f^2 is generous), which moves it by h times that; the new X itself is rounded (u f') and
summed ((K 2^-24) (|a| + |b| h^2 + |c| h^4) f). What one step leaves, later ones carry on with the iteration's
derivative, at most L = max |a + 3 b s^2 + 5 c s^4| or max |a + b s^2 + c s^4|, whichever is more."""
import numpy as np
import pytest
import torch

import oracle
import paper_2005_10761_amd as rt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"pairs": 2.0 ** -22, "halves": 2.0 ** -11}
OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
QUINTIC = [rt.QUINTIC] * 5


def reference(g, coefficients=QUINTIC, eps=1e-7, products="pairs"):
    """(result in binary64, room for its error in the Frobenius norm)"""
    g = np.asarray(g, np.float64)
    over = g.shape[0] > g.shape[1]
    x = g.T if over else g
    norm = np.sqrt((x * x).sum())
    x = x / (norm + eps) if norm else x
    u, sum_m, sum_n = UNIT[products], x.shape[0] * 2.0 ** -24, x.shape[1] * 2.0 ** -24
    room, h = u * np.sqrt((x * x).sum()), 1.0
    for a, b, c in coefficients:
        f = np.sqrt((x * x).sum())
        s = np.linspace(0, h, 2000)
        slope = max(np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max(), np.abs(a + b * s ** 2 + c * s ** 4).max())
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
        made = (u + sum_n) * f * f * (abs(b) * h + 2 * abs(c) * h ** 3) + (u + 2 * sum_m) * (abs(b) + abs(c) * h * h) * f * f * h
        made += u * np.sqrt((x * x).sum()) + sum_m * (abs(a) + abs(b) * h * h + abs(c) * h ** 4) * f
        room = room * slope + made
        h = np.abs(a * s + b * s ** 3 + c * s ** 5).max()
    return (x.T if over else x), room


def gradient(rng, rows, cols):
    rank = min(4, rows, cols)
    return (rng.standard_normal((rows, rank)) @ rng.standard_normal((rank, cols)) + rng.standard_normal((rows, cols))).astype(np.float32)


def laid(values, dtype, ld, offset=0, fill=7.0):
    rows, cols = values.shape
    store = torch.full((offset + rows * ld + 16,), fill, dtype=dtype, device=DEV)
    view = store[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.as_tensor(np.ascontiguousarray(values)).to(DEV).to(dtype))
    return view


def host(t):
    return t.detach().double().cpu().numpy()


def check(out, want, room, kind, sharp=None):
    got = host(out)
    off = np.sqrt(((got - want) ** 2).sum())
    size = np.sqrt((want ** 2).sum())
    room = room + OUT[kind] * size + 1e-7 * np.sqrt(want.size) * (kind == "f16")
    assert off <= room, (off, room, size)
    if sharp is not None:
        assert off <= (sharp + OUT[kind]) * size, (off / size, sharp)


# what the two forms of products promise for matrices of gradients: binary32's own error on this iteration, and half of bfloat16's step
SHARP = {"pairs": 2e-5, "halves": 2.0 ** -8}


@pytest.mark.parametrize("products", ["pairs", "halves"])
@pytest.mark.parametrize("rows, cols", [
    (1, 1), (1, 5), (5, 1), (2, 2), (3, 70), (70, 3), (16, 16), (31, 33), (33, 31), (64, 64), (64, 576), (65, 129), (576, 64), (100, 300),
    (128, 128), (129, 640), (130, 127), (257, 500), (600, 200), (700, 710), (1030, 300)])
def test_against_binary64(rows, cols, products):
    rng = np.random.default_rng(rows * 1009 + cols)
    g = gradient(rng, rows, cols)
    x = torch.as_tensor(g, device=DEV)
    out = torch.full((rows, cols), float("nan"), device=DEV)
    rt.orthogonalize([x], [out], products=products)
    want, room = reference(g, products=products)
    check(out, want, room, "f32", SHARP[products] if min(rows, cols) > 3 else None)
    assert np.array_equal(host(x), g.astype(np.float64))


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("out_kind", ["bf16", "f16", "f32"])
def test_types_row_distances_and_members(kind, out_kind):
    """Members of a batch of 17 (more than a launch holds) have nothing to do with each other."""
    rng = np.random.default_rng(5)
    for rows, cols, count, pad in ((40, 90, 17, 3), (90, 40, 3, 4), (130, 200, 2, 1)):
        gs = [gradient(rng, rows, cols) * 10.0 ** rng.uniform(-3, 3) for _ in range(count)]
        xs = [laid(g, TYPES[kind], cols + pad, 1) for g in gs]
        outs = [laid(np.zeros((rows, cols), np.float32), TYPES[out_kind], cols + pad + 1, i % 2) for i in range(count)]
        rt.orthogonalize(xs, outs)
        products = "halves" if out_kind == "bf16" else "pairs"
        for x, out in zip(xs, outs):
            want, room = reference(host(x), products=products)
            check(out, want, room, out_kind, SHARP[products])
            beyond = torch.as_strided(out, (rows - 1, pad + 1), (cols + pad + 1, 1), out.storage_offset() + cols)
            assert bool((beyond == 7).all())


def test_in_place_and_same_bits_again():
    rng = np.random.default_rng(6)
    g = torch.as_tensor(gradient(rng, 300, 140), device=DEV)
    first, second = torch.empty_like(g), torch.empty_like(g)
    rt.orthogonalize([g], [first])
    space = torch.empty(rt.orthogonalize_workspace_bytes(1, 300, 140), dtype=torch.uint8, device=DEV)
    space.fill_(0xA5)
    rt.orthogonalize([g], [second], workspace=space)
    assert torch.equal(first, second)
    # a member of a batch is computed as it is alone, whatever the batch
    other = torch.randn_like(g)
    a, b = torch.empty_like(g), torch.empty_like(g)
    rt.orthogonalize([other, g], [a, b])
    assert float((b - first).norm() / first.norm()) < 2e-5
    rt.orthogonalize([g], [g])
    assert torch.equal(g, first)


@pytest.mark.parametrize("coefficients", [
    [(1.5, -0.5, 0.0)] * 8, [(1.875, -1.25, 0.375)] * 6, [(2.0, -1.5, 0.5)], [(4.0, -7.0, 4.0), (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)],
    [(1.0, 0.0, 0.0)], [(0.0, 1.0, 0.0)], [(0.0, 0.0, 1.0)]])
def test_other_coefficients(coefficients):
    g = gradient(np.random.default_rng(7), 90, 200)
    x, out = torch.as_tensor(g, device=DEV), torch.empty(90, 200, device=DEV)
    rt.orthogonalize([x], [out], coefficients=coefficients)
    check(out, *reference(g, coefficients), "f32")


@pytest.mark.parametrize("products", ["pairs", "halves"])
@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-10, 1.0, 1e10, 1e30, 3e36])
def test_sizes_of_numbers(size, products):
    """The norm is taken out exactly, whatever the size; eps matters where the matrix is as small as it."""
    g = (gradient(np.random.default_rng(8), 70, 150) * np.float32(size)).astype(np.float32)
    x, out = torch.as_tensor(g, device=DEV), torch.empty(70, 150, device=DEV)
    for eps in (0.0, 1e-7):
        rt.orthogonalize([x], [out], eps=eps, products=products)
        want, room = reference(g, eps=float(np.float32(eps)), products=products)
        if size * 200 < eps * 1e-3:                 # nothing but eps: what is left is too small for halves
            assert float(out.abs().max()) < 1e-4
        else:
            check(out, want, room, "f32", SHARP[products])


def test_zeros_infinities_and_nans_stay_where_they_are():
    rng = np.random.default_rng(9)
    good = gradient(rng, 100, 140)
    inf, nan = good.copy(), good.copy()
    inf[3, 7], nan[99, 139] = np.inf, np.nan
    rows_out = good.copy()
    rows_out[10:40] = 0                             # a mask that leaves rows empty
    rows_out[:, 100:] = 0
    xs = [torch.as_tensor(v, device=DEV) for v in (np.zeros_like(good), inf, good, nan, rows_out)]
    for products in ("pairs", "halves"):
        for eps in (0.0, 1e-7):
            outs = [torch.full((100, 140), 5.0, device=DEV) for _ in xs]
            rt.orthogonalize(xs, outs, eps=eps, products=products)
            assert bool((outs[0] == 0).all())
            assert bool(torch.isnan(outs[1]).all()) and bool(torch.isnan(outs[3]).all())
            check(outs[2], *reference(good, products=products), "f32", SHARP[products])
            check(outs[4], *reference(rows_out, products=products), "f32", SHARP[products])
            assert bool((outs[4][10:40] == 0).all()) and bool((outs[4][:, 100:] == 0).all())


def test_another_stream_and_a_graph():
    g = torch.Generator(device=DEV).manual_seed(4)
    x, out, other = torch.randn(200, 330, device=DEV, generator=g), torch.empty(200, 330, device=DEV), torch.empty(200, 330, device=DEV)
    space = torch.empty(rt.orthogonalize_workspace_bytes(1, 200, 330), dtype=torch.uint8, device=DEV)
    rt.orthogonalize([x], [out], workspace=space)
    first = out.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    rt.orthogonalize([x], [other], stream=stream)
    stream.synchronize()
    assert torch.equal(first, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rt.orthogonalize([x], [out], workspace=space)
    for step in range(3):
        x.copy_(torch.randn(200, 330, device=DEV, generator=g))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        rt.orthogonalize([x], [other])
        assert torch.equal(out, other), step


@pytest.mark.parametrize("products", ["pairs", "halves"])
@pytest.mark.parametrize("rows, cols, count, n, k, nesterov", [
    (64, 576, 4, 5, 37, True), (1, 1, 1, 1, 1, True), (300, 70, 2, 3, 21, False), (129, 260, 1, 70, 33, True), (45, 45, 18, 2, 2025, False),
    (3, 5000, 1, 4, 15, True)])
def test_master_step(rows, cols, count, n, k, nesterov, products):
    rng = np.random.default_rng(rows + cols + n)
    d = rows * cols
    eta, scale, mu, decay, gain = 0.05, 1.5, 0.9, 0.1, 0.8
    idx = [np.stack([np.sort(rng.choice(d, k, replace=False)) for _ in range(n)]).astype(np.uint32) for _ in range(count)]
    val = [rng.standard_normal((n, k)).astype(np.float32) for _ in range(count)]
    w0 = [rng.standard_normal((rows, cols)).astype(np.float32) for _ in range(count)]
    v0 = [gradient(rng, rows, cols) for _ in range(count)]
    dev = lambda a: torch.as_tensor(a, device=DEV)      # noqa: E731
    omega, velocity = [dev(w.copy()) for w in w0], [dev(v.copy()) for v in v0]
    rt.aggregate_update_orthogonal([dev(i.reshape(-1).view(np.int32)) for i in idx], [dev(v.reshape(-1)) for v in val], n, k, eta, scale,
                                   mu, omega, velocity, nesterov=nesterov, decay=decay, gain=gain, products=products)
    f32 = np.float32
    for i in range(count):
        average = oracle.aggregate_f32(idx[i].reshape(-1), val[i].reshape(-1), n, d).reshape(rows, cols)
        u = (f32(scale) * average).astype(f32)
        v = (float(f32(mu)) * v0[i].astype(np.float64) + u).astype(f32)          # one rounding (binary64 holds the product and sum)
        assert np.abs(host(velocity[i]) - v).max() <= 2.0 ** -23 * np.abs(v).max()
        g = (float(f32(mu)) * v.astype(np.float64) + u).astype(f32) if nesterov else v
        want, room = reference(g, products=products)
        step, keep = eta * gain, 1 - eta * decay
        moved = keep * w0[i].astype(np.float64) - step * want
        got = host(omega[i])
        room = step * min(room + 1e-6, (SHARP[products] if min(rows, cols) > 3 else 1.0) * np.sqrt((want ** 2).sum()) + 1e-6)
        room += 2.0 ** -22 * np.sqrt((w0[i].astype(np.float64) ** 2).sum())
        assert np.sqrt(((got - moved) ** 2).sum()) <= room


def test_refusals_of_the_binding():
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)     # noqa: E731
    with pytest.raises(TypeError):
        rt.orthogonalize([z(4, 6).t()], [z(6, 4)])
    with pytest.raises(TypeError):
        rt.orthogonalize([z(4, 6, t=torch.float64)], [z(4, 6)])
    with pytest.raises(TypeError):
        rt.orthogonalize([z(4, 6), z(4, 6, t=torch.bfloat16)], [z(4, 6), z(4, 6)])
    with pytest.raises(ValueError):
        rt.orthogonalize([z(4, 6), z(4, 7)], [z(4, 6), z(4, 7)])
    with pytest.raises(ValueError):
        rt.orthogonalize([z(4, 6)], [z(4, 6), z(4, 6)])
    with pytest.raises(ValueError):
        rt.orthogonalize([z(4, 6)], [z(4, 6)], coefficients=(1.5, -0.5))
    with pytest.raises(KeyError):
        rt.orthogonalize([z(4, 6)], [z(4, 6)], products="singles")
    for bad in (dict(coefficients=(9.0, 0.0, 0.0)), dict(eps=-1.0), dict(steps=0)):
        with pytest.raises((rt.RtopkError, ValueError)):
            rt.orthogonalize([z(4, 6)], [z(4, 6)], **bad)
    with pytest.raises(ValueError):
        rt.aggregate_update_orthogonal([z(4, t=torch.int32)], [z(4)], 2, 3, 0.1, 1.0, 0.9, [z(4, 6)], [z(4, 6)])
    with pytest.raises(ValueError):
        rt.aggregate_update_orthogonal([z(6, t=torch.int32)], [z(6)], 2, 3, 0.1, 1.0, 0.9, [z(4, 6)], [z(4, 5)])
