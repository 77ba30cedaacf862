"""4-bit quantisation, products and a layer's forward and backward on the GPU, against the definitions: numbers and
scales bit for bit, sums that are whole multiples of 1/4 below 2^22 exactly, other sums within what the steps of a
binary32 accumulation round."""
import numpy as np
import pytest
import torch

import paper_2005_10761_amd as rt
from tests import four_bits as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 1e-40), "f16": (2.0 ** -11, 2.0 ** -25)}


def laid(values, dtype, ld=None, offset=0, fill=77):
    """A device matrix whose rows are `ld` elements apart and which starts `offset` elements into its storage; what lies
    between is garbage that must not matter."""
    rows, cols = values.shape
    ld = cols if ld is None else ld
    store = torch.full((offset + rows * ld + 64,), fill, dtype=dtype, device=DEV)
    view = store[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.as_tensor(np.ascontiguousarray(values)).to(DEV).to(dtype))
    return view


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def room_for(rows, k, pad=0, scale_pad=0, offset=0):
    """Memory for a quantised matrix, filled with 99, and its stores."""
    have, blocks = (k + 1) // 2, fb.blocks_of(k)
    q_store = torch.full((offset + rows * (have + pad) + 16,), 99, dtype=torch.uint8, device=DEV)
    s_store = torch.full((offset + blocks * (rows + scale_pad) + 16,), 99, dtype=torch.uint8, device=DEV)
    q = q_store[offset:offset + rows * (have + pad)].view(rows, have + pad)
    s = s_store[offset:offset + blocks * (rows + scale_pad)].view(blocks, rows + scale_pad)
    return q[:, :have], s[:, :rows], (q_store, s_store)


def untouched(view, store, offset):
    """Whether all of the store outside of the view still is 99."""
    mask = torch.ones_like(store, dtype=torch.bool)
    mask[offset:offset + view.shape[0] * view.stride(0)].view(view.shape[0], view.stride(0))[:, :view.shape[1]] = False
    return bool((store[mask] == 99).all())


def operand(rng, rows, k, low=127, high=127, pad=0, scale_pad=0, offset=0):
    """A random quantised matrix: (numbers, scale bytes, device q, device scale)."""
    q, s = rng.integers(0, 16, (rows, k)).astype(np.uint8), rng.integers(low, high + 1, (fb.blocks_of(k), rows)).astype(np.uint8)
    have = (k + 1) // 2
    return q, s, laid(fb.packed(q), torch.uint8, have + pad, offset, fill=255), laid(s, torch.uint8, rows + scale_pad, offset, fill=255)


def check(out, kind, a, b, bias=None, exact=False):
    """out against a b^T + bias in binary64."""
    want = a @ b.T + (0.0 if bias is None else bias.astype(np.float64))
    rel, least = ROUND[kind]
    if exact:
        room = np.zeros_like(want)
    else:
        # each instruction of 128 products, and each of up to 16 runs' sums, is off by less than 4 units in the last place of the
        # magnitudes that it adds
        size = np.abs(a) @ np.abs(b).T
        room = 2.0 ** -21 * (a.shape[1] / 128 + 18) * size
    room = room + (0.0 if bias is None else 2.0 ** -23 * (np.abs(want) + np.abs(bias)))
    room = room + rel * (np.abs(want) + room) + least
    got = host(out)
    assert got.shape == want.shape
    if kind == "f16":
        beyond = np.abs(want) >= 65520
        close = np.abs(np.abs(want) - 65520) <= 2 * room
        assert np.all((np.isinf(got) & (np.sign(got) == np.sign(want)))[beyond & ~close])
        got, want, room = got[~beyond & ~close], want[~beyond & ~close], room[~beyond & ~close]
    off = ~(np.abs(got - want) <= room)
    assert not off.any(), (int(off.sum()), np.argwhere(off)[:4], got[off][:4], want[off][:4], room[off][:4])


SIZES = [(1, 1, 0, 0), (1, 1500, 0, 0), (3, 7, 1, 1), (5, 32, 0, 0), (64, 129, 3, 1), (130, 511, 1, 0), (1030, 40, 0, 0),
         (300, 1052, 4, 3), (7, 5000, 0, 0), (33, 64, 8, 8), (257, 96, 0, 0), (16, 31, 0, 0), (700, 65, 7, 5)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, cols, pad, offset", SIZES)
def test_numbers_and_scales(kind, rows, cols, pad, offset):
    rng = np.random.default_rng(rows * 10_007 + cols)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    x[rng.random((rows, cols)) < 0.1] = 0
    x[rng.random((rows, cols)) < 0.05] = -0.0
    if rows > 4:
        x[1] = 0
        x[2] = rng.integers(-28, 29, cols) / 4              # the numbers, the ties between them, and 7
        x[3] = np.where(rng.random(cols) < 0.5, 6.0, 7.0)
    xd = laid(x, TYPES[kind], cols + pad, offset)
    x = host(xd)
    for along in ("rows", "columns"):
        for seed, step in ((None, 0), (42, 7), (2 ** 63 + 5, 2 ** 40 + 3)):
            want_q, want_s = fb.quantized(x, along, seed, step)
            r, c = want_q.shape
            for q_pad, s_pad, at in ((0, 0, 0), (5, 3, 1), (-(c + 1) // 2 % 16 + 16, -r % 16 + 16, 0)):
                q, s, (q_store, s_store) = room_for(r, c, q_pad, s_pad, at)
                rt.quantize_mx4(xd, q, s, along=along, seed=seed, step=step)
                assert np.array_equal(host(s), want_s), (along, seed)
                assert np.array_equal(host(q), fb.packed(want_q)), (along, seed)
                assert untouched(q, q_store, at) and untouched(s, s_store, at)
            for out_kind in ("f32", kind):
                out = torch.full((r, c + 3), 5.0, dtype=TYPES[out_kind], device=DEV)
                rt.dequantize_mx4(q, s, out[:, :c])
                exact = torch.as_tensor(fb.values(want_q, want_s)).to(TYPES[out_kind])
                assert torch.equal(out[:, :c].cpu(), exact) and bool((out[:, c:] == 5).all())


def test_blocks_without_numbers_and_at_the_ends_of_the_range():
    cols = 100
    x = np.ones((10, cols), np.float32)
    x[0, 5] = np.nan
    x[1, 99] = np.inf
    x[2, 32] = -np.inf
    x[3] = 0
    x[4] = 1e-40
    x[5] = 2.0 ** -126
    x[6] = 3.4028235e38
    x[7] = -0.0
    x[8, ::2] = 1e-45
    x[9, 1] = 1e38
    xd = laid(x, torch.float32)
    for along in ("rows", "columns"):
        for seed in (None, 9):
            want_q, want_s = fb.quantized(x, along, seed, 1)
            q, s, _ = room_for(*want_q.shape)
            rt.quantize_mx4(xd, q, s, along=along, seed=seed, step=1)
            assert np.array_equal(host(s), want_s) and np.array_equal(host(q), fb.packed(want_q)), (along, seed)
    # through a layer: NaN rows come out as NaN, rows of zeros as the bias
    rng = np.random.default_rng(0)
    wq, ws, wqd, wsd = operand(rng, 120, cols, 120, 130)
    bias = np.linspace(-1, 1, 120).astype(np.float32)
    out = torch.empty(10, 120, device=DEV)
    rt.linear_mx4(xd, wqd, wsd, out, bias=torch.as_tensor(bias, device=DEV))
    got = host(out)
    assert np.isnan(got[:3]).all() and not np.isnan(got[3:6]).any()
    assert np.array_equal(got[3], bias.astype(np.float64)) and np.array_equal(got[7], bias.astype(np.float64))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_every_16_bit_number(kind):
    """All of them but infinities and not-a-numbers, each by itself in a block with 1.5 2^e, and in blocks that a subnormal leads."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[kind])
    every = every[torch.isfinite(every)]
    for lead in (1.5, 6.0, 2.0 ** -10, 2.0 ** -24) + ((1.5 * 2.0 ** -124, 2.0 ** -126, 2.0 ** -130) if kind == "bf16" else ()):
        few = every[every.abs().double() <= lead]
        x = few[torch.randperm(len(few), generator=torch.Generator().manual_seed(1))]
        x = torch.nn.functional.pad(x, (0, -len(x) % 31)).view(-1, 31)
        x = torch.cat([torch.full((len(x), 1), lead, dtype=TYPES[kind]), x], 1).to(DEV)
        for along, given in (("rows", x), ("columns", x.T.contiguous())):
            for seed in (None, 1, 2):
                want_q, want_s = fb.quantized(host(given), along, seed, 5)
                q, s, _ = room_for(*want_q.shape)
                rt.quantize_mx4(given, q, s, along=along, seed=seed, step=5)
                assert np.array_equal(host(s), want_s) and np.array_equal(host(q), fb.packed(want_q)), (lead, along, seed)


def test_drawn_rounding_keeps_the_mean():
    x = torch.linspace(-6, 6, 64, device=DEV).repeat(64, 1)
    q, s, _ = room_for(64, 64)
    out, total = torch.empty_like(x), torch.zeros(64, device=DEV, dtype=torch.float64)
    for step in range(200):
        rt.quantize_mx4(x, q, s, seed=5, step=step)
        rt.dequantize_mx4(q, s, out)
        total += out.double().mean(0)
    # 12,800 draws a column; a step is 2 at most: a deviation of at most 1 / sqrt(12800)
    assert float((total / 200 - x[0].double()).abs().max()) < 6 / 12_800 ** 0.5


PRODUCTS = [(1, 1, 1), (2, 3, 15), (15, 17, 33), (16, 16, 128), (17, 100, 127), (33, 65, 256), (64, 64, 257), (100, 130, 500),
            (129, 257, 640), (300, 70, 1500), (257, 513, 1024), (40, 48, 20_000), (13, 1000, 777), (1, 4096, 4096), (200, 3000, 96)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_products(kind, m, n, k):
    rng = np.random.default_rng(m * 1009 + n * 31 + k)
    bias = rng.standard_normal(n).astype(np.float32)
    bd = torch.as_tensor(bias, device=DEV)
    for low, high, pads in ((127, 127, (0, 0, 0)), (110, 135, (0, 0, 0)), (127, 127, (5, 3, 1)), (120, 130, (-(k + 1) // 2 % 16, 16, 0))):
        aq, as_, ad, asd = operand(rng, m, k, low, high, pads[0], -m % 16 + 16 if pads[1] == 16 else pads[1], pads[2])
        bq, bs, bqd, bsd = operand(rng, n, k, low, high, pads[0], -n % 16 + 16 if pads[1] == 16 else pads[1], pads[2])
        a, b = fb.values(aq, as_), fb.values(bq, bs)
        store = torch.full((m, n + 5), 7.0, dtype=TYPES[kind], device=DEV)
        out = store[:, 1:1 + n]
        rt.matmul_mx4(ad, asd, bqd, bsd, out)
        check(out, kind, a, b, exact=low == high)
        rt.matmul_mx4(ad, asd, bqd, bsd, out, bias=bd)
        check(out, kind, a, b, bias)
        assert bool((store[:, 0] == 7).all()) and bool((store[:, 1 + n:] == 7).all())


def test_products_of_no_numbers():
    q, s = torch.empty(4, 0, dtype=torch.uint8, device=DEV), torch.empty(0, 4, dtype=torch.uint8, device=DEV)
    p, t = torch.empty(6, 0, dtype=torch.uint8, device=DEV), torch.empty(0, 6, dtype=torch.uint8, device=DEV)
    bias, out = torch.randn(6, device=DEV), torch.empty(4, 6, device=DEV)
    rt.matmul_mx4(q, s, p, t, out, bias=bias)
    assert torch.equal(out, bias.expand(4, 6))
    rt.matmul_mx4(q, s, p, t, out)
    assert not out.any()
    rt.dequantize_mx4(q, s, torch.empty(4, 0, device=DEV))


def test_product_without_terms_is_the_bias():
    lib = rt.load_library()
    bias, out = torch.randn(10, device=DEV), torch.empty(4, 10, device=DEV)
    rc = lib.rtopk_matmul_mx4(None, None, None, None, bias.data_ptr(), 4, 10, 0, 0, 4, 0, 10, out.data_ptr(), 0, 10, None, 0, None)
    torch.cuda.synchronize()
    assert rc == 0 and torch.equal(out, bias.expand(4, 10))


@pytest.mark.parametrize("kind, out_kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("m, k, n", [(1, 1, 1), (1, 1500, 1000), (3, 33, 40), (13, 500, 70), (16, 512, 64), (17, 129, 300), (1, 9000, 20),
                                     (5, 2048, 3000), (16, 5000, 500), (100, 96, 80), (260, 1500, 300)])
def test_layer(kind, out_kind, m, k, n):
    rng = np.random.default_rng(m * 101 + k * 7 + n)
    xd = laid(rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1))), TYPES[kind], k + 3, 1)
    x = fb.values(*fb.quantized(host(xd)))
    wq, ws, wd, wsd = operand(rng, n, k, 118, 122, -(k + 1) // 2 % 16, -n % 16)
    w = fb.values(wq, ws)
    bias = rng.standard_normal(n).astype(np.float32)
    out = torch.full((m, n + 1), 3.0, dtype=TYPES[out_kind], device=DEV)
    rt.linear_mx4(xd, wd, wsd, out[:, :n], bias=torch.as_tensor(bias, device=DEV))
    check(out[:, :n], out_kind, x, w, bias)
    assert bool((out[:, n] == 3).all())
    rt.linear_mx4(xd, wd, wsd, out[:, :n])
    check(out[:, :n], out_kind, x, w)
    # one token by itself has the bits that it has among the others of a call that takes the same kernel
    if 1 < m <= 16:
        both, alone = torch.empty(m, n, device=DEV), torch.empty(1, n, device=DEV)
        rt.linear_mx4(xd, wd, wsd, both)
        rt.linear_mx4(xd[m - 1:], wd, wsd, alone)
        check(alone, "f32", x[m - 1:], w)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m, k, n", [(1, 1, 1), (2, 70, 33), (35, 64, 96), (100, 96, 80), (257, 130, 67), (512, 40, 300), (700, 150, 600)])
@pytest.mark.parametrize("seed", [None, 77])
def test_layer_backward(kind, m, k, n, seed):
    rng = np.random.default_rng(m * 11 + k * 3 + n)
    xd = laid(rng.standard_normal((m, k)), TYPES[kind], k + 1, 1)
    dyd = laid(rng.standard_normal((m, n)) * 0.01, TYPES[kind], n + 2, 2)
    wd = torch.as_tensor(rng.standard_normal((n, k)).astype(np.float32), device=DEV)
    turned, turned_scale, _ = room_for(k, n, -(n + 1) // 2 % 16, -k % 16)
    rt.quantize_mx4(wd, turned, turned_scale, along="columns")
    x, dy, w = host(xd), host(dyd), host(wd)
    dx = torch.full((m, k + 1), 3.0, dtype=TYPES[kind], device=DEV)
    dw, db = torch.full((n, k + 2), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV)
    rt.linear_mx4_backward(dyd, xd, turned, turned_scale, dx[:, :k], dw[:, :k], db, seed=seed, step=12)
    check(dx[:, :k], kind, fb.values(*fb.quantized(dy, "rows", seed, 12)), fb.values(*fb.quantized(w, "columns")))
    check(dw[:, :k], "f32", fb.values(*fb.quantized(dy, "columns", seed, 12)), fb.values(*fb.quantized(x, "columns")))
    assert bool((dx[:, k:] == 3).all()) and bool((dw[:, k:] == 3).all())
    # a sum of 256 rows in binary32 on the way, in any order, then binary64
    assert np.all(np.abs(host(db) - dy.sum(0)) <= 2.0 ** -24 * 258 * np.abs(dy).sum(0))
    alone_dx, alone_dw = torch.empty(m, k, dtype=TYPES[kind], device=DEV), torch.empty(n, k, device=DEV)
    rt.linear_mx4_backward(dyd, None, turned, turned_scale, alone_dx, None, seed=seed, step=12)
    rt.linear_mx4_backward(dyd, xd, None, None, None, alone_dw, seed=seed, step=12)
    assert torch.equal(alone_dx, dx[:, :k]) and torch.equal(alone_dw, dw[:, :k])


def test_no_tokens():
    e = lambda *s: torch.empty(*s, device=DEV)   # noqa: E731
    q, s, _ = room_for(8, 6)
    out, dw, db = e(0, 8), torch.full((8, 6), 3.0, device=DEV), torch.full((8,), 3.0, device=DEV)
    rt.linear_mx4(e(0, 6), q, s, out)
    rt.linear_mx4_backward(e(0, 8), e(0, 6), None, None, None, dw, db)
    assert not dw.any() and not db.any()


def test_gradients_are_those_of_the_quantised_product():
    """Against differences: where the quantised operands do not move, the layer is linear, and its gradients are exact."""
    rng = np.random.default_rng(3)
    m, k, n = 32, 64, 32
    # whole operands are numbers already: quantising them changes nothing
    pick = lambda *s: fb.VALUES[rng.integers(0, 16, s)].astype(np.float32)   # noqa: E731
    x, w, dy = pick(m, k), pick(n, k), pick(m, n)
    x[:, 0::32] = 6
    x[0::32] = 6
    w[:, 0::32] = w[0::32] = 6
    dy[:, 0::32] = dy[0::32] = 6
    xd, wd, dyd = (torch.as_tensor(v, device=DEV) for v in (x, w, dy))
    by_rows, row_scale, _ = room_for(n, k)
    by_cols, col_scale, _ = room_for(k, n)
    rt.quantize_mx4(wd, by_rows, row_scale)
    rt.quantize_mx4(wd, by_cols, col_scale, along="columns")
    dx, dw, db = torch.empty(m, k, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    rt.linear_mx4_backward(dyd, xd, by_cols, col_scale, dx, dw, db)

    def loss(x, w):
        wq, ws, _ = room_for(n, k)
        rt.quantize_mx4(w, wq, ws)
        y = torch.empty(m, n, device=DEV)
        rt.linear_mx4(x, wq, ws, y)
        return float((y.double() * dyd.double()).sum())

    base = loss(xd, wd)
    for i, j in ((0, 0), (5, 33), (31, 63)):
        # from one number to another that the block's scale has too
        moved = xd.clone()
        moved[i, j] = -moved[i, j] if moved[i, j] else 2.0
        assert loss(moved, wd) - base == float(moved[i, j] - xd[i, j]) * float(dx[i, j])
        moved = wd.clone()
        moved[i, j] = -moved[i, j] if moved[i, j] else 2.0
        assert loss(xd, moved) - base == float(moved[i, j] - wd[i, j]) * float(dw[i, j])
    assert torch.equal(db, dyd.sum(0))


def test_a_given_workspace_and_another_stream():
    rng = np.random.default_rng(5)
    m, k, n = 300, 700, 200
    xd = laid(rng.standard_normal((m, k)), torch.bfloat16)
    _, _, wd, wsd = operand(rng, n, k, 118, 122, 2, 8)
    want, got = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    rt.linear_mx4(xd, wd, wsd, want)
    need = rt.linear_mx4_workspace_bytes(m, k, n)
    store = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    at = -store.data_ptr() % 256
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    rt.linear_mx4(xd, wd, wsd, got, workspace=store[at:at + need], stream=stream)
    stream.synchronize()
    assert torch.equal(want, got) and bool((store[at + need:] == 255).all())
    with pytest.raises(rt.RtopkError) as e:
        rt.linear_mx4(xd, wd, wsd, got, workspace=store[at:at + need - 1])
    assert e.value.code == -2
