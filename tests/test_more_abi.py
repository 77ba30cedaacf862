"""Host-side argument checks of the 4-bit products, layer norm and dropout: what is refused is refused before anything is
launched, so no GPU is needed."""
import ctypes
import math

import pytest

import paper_2005_10761_amd as rt

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: checks fail first
FAKE2 = ctypes.c_void_p(0x10000000)
BIG = ctypes.c_uint64(1 << 40)
MOST = 1 << 22


def _with(call, **given):
    return lambda **k: call(*({**given, **k}.values()))


def _code(call):
    with pytest.raises(rt.RtopkError) as e:
        call()
    return e.value.code


def test_workspace_sizes_and_their_domains():
    assert rt.matmul_mx4_workspace_bytes(0, 5, 5) == 0 and rt.matmul_mx4_workspace_bytes(5, 5, 0) == 0
    assert rt.linear_mx4_workspace_bytes(0, 5, 5) == 0
    assert rt.linear_mx4_workspace_bytes(300, 130, 5) >= 300 * 65 + 300 * 5
    assert rt.linear_mx4_backward_workspace_bytes(0, 5, 5) == 0
    assert rt.linear_mx4_backward_workspace_bytes(100, 64, 96) >= (100 * 96 + 96 * 100 + 64 * 100) // 2
    assert rt.layer_norm_backward_workspace_bytes(0, 5) == 0 and rt.layer_norm_backward_workspace_bytes(2048, 1024) == 0
    assert rt.layer_norm_backward_workspace_bytes(3000, 5) >= 40
    for call in (lambda: rt.matmul_mx4_workspace_bytes(4, 4, MOST + 1), lambda: rt.matmul_mx4_workspace_bytes(MOST + 1, 4, 4),
                 lambda: rt.linear_mx4_workspace_bytes(4, 0, 4), lambda: rt.linear_mx4_workspace_bytes(4, 4, 0),
                 lambda: rt.linear_mx4_backward_workspace_bytes(4, 4, MOST + 1), lambda: rt.layer_norm_backward_workspace_bytes(4, 0),
                 lambda: rt.layer_norm_backward_workspace_bytes(MOST + 1, 4)):
        assert _code(call) == -1


def test_quantize_refusals():
    q = _with(rt.load_library().rtopk_quantize_mx4, x=FAKE, type=0, rows=4, cols=40, ldx=40, along=0, rounding=0, seed=0, step=0, at=None,
              q=FAKE2, ldq=20, scale=FAKE, lds=4, stream=None)
    for bad in (dict(x=None), dict(type=3), dict(type=-1), dict(ldx=39), dict(ldq=19), dict(lds=3), dict(along=2), dict(rounding=2),
                dict(q=None), dict(scale=None), dict(rows=MOST + 1, lds=MOST + 1), dict(cols=0), dict(cols=MOST + 1, ldx=MOST + 1),
                dict(ldx=MOST + 1), dict(ldq=MOST + 1), dict(lds=MOST + 1), dict(along=1, ldq=1, lds=40), dict(along=1, ldq=2, lds=39)):
        assert q(**bad) == -1, bad
    assert q(rows=0, x=None, q=None, scale=None) == 0
    back = _with(rt.load_library().rtopk_dequantize_mx4, q=FAKE, rows=4, cols=41, ldq=21, scale=FAKE, lds=4, out=FAKE2, type=0, ldo=41,
                 stream=None)
    for bad in (dict(q=None), dict(scale=None), dict(out=None), dict(type=9), dict(ldq=20), dict(lds=3), dict(ldo=40), dict(ldo=MOST + 1),
                dict(rows=MOST + 1, lds=MOST + 1)):
        assert back(**bad) == -1, bad
    assert back(rows=0, q=None, scale=None, out=None) == 0 and back(cols=0, q=None, out=None) == 0


def test_product_and_layer_refusals():
    lib = rt.load_library()
    mm = _with(lib.rtopk_matmul_mx4, a=FAKE, sa=FAKE, b=FAKE, sb=FAKE, bias=None, m=4, n=6, k=40, lda=20, ldsa=4, ldb=20, ldsb=6,
               out=FAKE2, type=0, ldo=6, ws=FAKE, bytes=BIG, stream=None)
    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(out=None), dict(lda=19), dict(ldsa=3), dict(ldb=19),
                dict(ldsb=5), dict(ldo=5), dict(type=3), dict(k=MOST + 1), dict(lda=MOST + 1), dict(ldsb=MOST + 1), dict(m=MOST + 1, ldsa=MOST + 1)):
        assert mm(**bad) == -1, bad
    assert mm(m=0, a=None) == 0 and mm(n=0, b=None) == 0
    fw = _with(lib.rtopk_linear_mx4, x=FAKE, type=0, m=400, k=800, ldx=800, w=FAKE, ws=FAKE, n=400, ldw=400, lds=400, bias=None, out=FAKE2,
               out_type=0, ldo=400, room=FAKE, bytes=BIG, stream=None)
    for bad in (dict(x=None), dict(w=None), dict(ws=None), dict(out=None), dict(type=3), dict(out_type=-1), dict(ldx=799), dict(ldw=399),
                dict(lds=399), dict(ldo=399), dict(k=0), dict(n=0, lds=400), dict(m=MOST + 1)):
        assert fw(**bad) == -1, bad
    need = rt.linear_mx4_workspace_bytes(400, 800, 400)
    assert need > 0
    assert fw(room=None) == -2 and fw(bytes=need - 1) == -2 and fw(room=ctypes.c_void_p(0x1010)) == -2
    assert fw(m=0, x=None, w=None, ws=None, out=None) == 0
    bw = _with(lib.rtopk_linear_mx4_backward, dy=FAKE, x=FAKE, type=0, m=4, k=8, n=6, lddy=6, ldx=8, w=FAKE, s=FAKE, ldw=3, lds=8,
               rounding=1, seed=1, step=2, at=None, dx=FAKE2, lddx=8, dw=FAKE2, lddw=8, db=FAKE2, ws=FAKE, bytes=BIG, stream=None)
    for bad in (dict(dy=None), dict(x=None), dict(w=None), dict(s=None), dict(type=7), dict(lddy=5), dict(ldx=7), dict(ldw=2), dict(lds=7),
                dict(lddx=7), dict(lddw=7), dict(dx=None, dw=None), dict(dw=None), dict(rounding=-1), dict(k=0), dict(n=0),
                dict(lddy=MOST + 1), dict(ldx=MOST + 1)):
        assert bw(**bad) == -1, bad
    assert bw(ws=None) == -2 and bw(bytes=8) == -2
    assert bw(m=0, dy=None, dw=None, db=None, ws=None) == 0


def test_norm_refusals():
    lib = rt.load_library()
    fw = _with(lib.rtopk_layer_norm, x=FAKE, type=0, rows=4, cols=40, ldx=40, gamma=None, beta=None, eps=ctypes.c_float(1e-5), out=FAKE2,
               out_type=1, ldo=40, mean=None, rstd=None, stream=None)
    for bad in (dict(x=None), dict(out=None), dict(type=3), dict(out_type=-1), dict(ldx=39), dict(ldo=39), dict(cols=0), dict(rows=MOST + 1),
                dict(ldx=MOST + 1), dict(eps=ctypes.c_float(-1e-5)), dict(eps=ctypes.c_float(math.nan)), dict(eps=ctypes.c_float(math.inf)),
                dict(out=FAKE), dict(out=FAKE, out_type=0, ldo=41)):
        assert fw(**bad) == -1, bad
    assert fw(rows=0, x=None, out=None) == 0
    bw = _with(lib.rtopk_layer_norm_backward, dy=FAKE, dy_type=1, x=FAKE, type=0, rows=4, cols=40, lddy=40, ldx=40, mean=FAKE, rstd=FAKE,
               gamma=None, add=None, ldadd=0, dx=FAKE2, lddx=40, dgamma=FAKE2, dbeta=FAKE2, ws=FAKE, bytes=BIG, stream=None)
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dy_type=3), dict(type=-1), dict(lddy=39), dict(ldx=39),
                dict(lddx=39), dict(dx=None, dgamma=None, dbeta=None), dict(add=FAKE, ldadd=39), dict(add=FAKE, ldadd=40, dx=None),
                dict(cols=0), dict(rows=MOST + 1), dict(dx=FAKE, dy=FAKE2, lddx=41), dict(dx=FAKE, x=FAKE2), dict(dx=FAKE, add=FAKE, x=FAKE2,
                                                                                                                  dy=FAKE2, ldadd=44)):
        assert bw(**bad) == -1, bad
    large = dict(rows=4000)
    assert bw(**large, ws=None) == -2 and bw(**large, bytes=8) == -2 and bw(**large, ws=ctypes.c_void_p(0x1010)) == -2


def test_dropout_refusals():
    d = _with(rt.load_library().rtopk_dropout, x=FAKE, type=0, rows=4, cols=40, ldx=40, residual=None, ldr=0, out=FAKE2, out_type=0, ldo=40,
              p=ctypes.c_double(0.5), seed=1, step=2, at=None, stream=None)
    for bad in (dict(x=None), dict(out=None), dict(type=3), dict(out_type=-1), dict(ldx=39), dict(ldo=39), dict(residual=FAKE, ldr=39),
                dict(p=ctypes.c_double(-0.1)), dict(p=ctypes.c_double(1.1)), dict(p=ctypes.c_double(math.nan)), dict(rows=1 << 32),
                dict(rows=1 << 20, cols=(1 << 20) + 1, ldx=1 << 21, ldo=1 << 21), dict(ldx=1 << 32), dict(out=FAKE, out_type=1),
                dict(out=FAKE, ldo=41), dict(residual=FAKE2, ldr=41)):
        assert d(**bad) == -1, bad
    assert d(rows=0, x=None, out=None) == 0 and d(cols=0, x=None, out=None) == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    x, q = torch.zeros(4, 8), torch.zeros(4, 4, dtype=torch.uint8)
    for call in (lambda: rt.quantize_mx4(x, q, q), lambda: rt.dequantize_mx4(q, q, x), lambda: rt.matmul_mx4(q, q, q, q, x),
                 lambda: rt.linear_mx4(x, q, q, x), lambda: rt.layer_norm(x, None, None, x),
                 lambda: rt.layer_norm_backward(x, x, x, x, None, x), lambda: rt.dropout(x, x, 0.5, 1, 2),
                 lambda: rt.linear_mx4_backward(x, x, q, q, x, x)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rt.linear_mx4_backward(x, x, q, q, None, None), lambda: rt.linear_mx4_backward(x, x, None, None, x, None),
                 lambda: rt.linear_mx4_backward(x, None, q, q, None, x), lambda: rt.linear_mx4_backward(x, x, q, q, x, None, db=x),
                 lambda: rt.layer_norm_backward(x, x, x, x, None, None), lambda: rt.layer_norm_backward(x, x, x, x, None, None, x, add=x)):
        with pytest.raises(ValueError):
            call()
