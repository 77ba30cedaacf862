"""Host-side argument checks of the matrix entry points (8-bit products, orthogonalised updates): what is refused is
refused before anything is launched, so no GPU is needed; and the workspace sizes that the host computes."""
import ctypes
import math

import pytest

import paper_2005_10761_amd as rt

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: checks fail first
FAKE2 = ctypes.c_void_p(0x10000000)
BIG = ctypes.c_uint64(1 << 40)
MOST = 1 << 22


def _code(call):
    with pytest.raises(rt.RtopkError) as e:
        call()
    return e.value.code


def test_workspace_sizes_and_their_domains():
    assert rt.quantize_i8_workspace_bytes(10, 20) == 0
    assert rt.quantize_i8_workspace_bytes(10, 20, "columns") == 256
    assert rt.quantize_i8_workspace_bytes(0, 20, "columns") == 0
    assert rt.matmul_i8_workspace_bytes(0, 5, 5) == 0 and rt.matmul_i8_workspace_bytes(5, 5, 0) == 0
    assert rt.linear_i8_workspace_bytes(0, 5, 5) == 0
    assert rt.linear_i8_workspace_bytes(100, 130, 5) >= 100 * 256 + 100 * 4
    assert rt.linear_i8_workspace_bytes(1, 1500, 10_000) == 0       # one launch, nothing kept
    assert rt.linear_i8_backward_workspace_bytes(0, 5, 5) == 0
    one = rt.orthogonalize_workspace_bytes(1, 100, 300, "halves")
    assert one >= 4 * 100 * 300 * 2 + 2 * 100 * 100 * 2
    assert rt.orthogonalize_workspace_bytes(1, 300, 100, "halves") == one
    assert rt.orthogonalize_workspace_bytes(1, 100, 300, "pairs") > one
    assert rt.orthogonalize_workspace_bytes(16, 100, 300, "halves") <= rt.orthogonalize_workspace_bytes(40, 100, 300, "halves") < 17 * one
    assert rt.aggregate_update_orthogonal_workspace_bytes(1, 100, 300, "halves") >= one + 4 * 100 * 300
    for call in (lambda: rt.quantize_i8_workspace_bytes(MOST + 1, 4), lambda: rt.quantize_i8_workspace_bytes(4, 0),
                 lambda: rt.matmul_i8_workspace_bytes(4, 4, MOST + 1), lambda: rt.linear_i8_workspace_bytes(4, 0, 4),
                 lambda: rt.linear_i8_workspace_bytes(4, 4, 0), lambda: rt.linear_i8_backward_workspace_bytes(4, 4, MOST + 1),
                 lambda: rt.orthogonalize_workspace_bytes(0, 4, 4), lambda: rt.orthogonalize_workspace_bytes(1, 0, 4),
                 lambda: rt.orthogonalize_workspace_bytes(1, 4, (1 << 21) + 1),
                 lambda: rt.orthogonalize_workspace_bytes(1, 1 << 17, 1 << 17),
                 lambda: rt.aggregate_update_orthogonal_workspace_bytes(1, 1 << 16, 1 << 16)):
        assert _code(call) == -1


def test_quantize_refusals():
    q = rt.load_library().rtopk_quantize_i8
    assert q(None, 0, 4, 8, 8, 0, FAKE, 8, FAKE, None, 0, None) == -1
    assert q(FAKE, 3, 4, 8, 8, 0, FAKE2, 8, FAKE, None, 0, None) == -1          # no such type
    assert q(FAKE, 0, 4, 8, 7, 0, FAKE2, 8, FAKE, None, 0, None) == -1          # rows overlap
    assert q(FAKE, 0, 4, 8, 8, 0, FAKE2, 7, FAKE, None, 0, None) == -1
    assert q(FAKE, 0, 4, 8, 8, 1, FAKE2, 3, FAKE, FAKE, BIG, None) == -1        # turned over: rows of 4
    assert q(FAKE, 0, 4, 8, 8, 2, FAKE2, 8, FAKE, None, 0, None) == -1          # along neither
    assert q(FAKE, 0, 4, 8, 8, 0, FAKE2, 8, None, None, 0, None) == -1
    assert q(FAKE, 0, 4, 8, 8, 1, FAKE2, 4, FAKE, None, 0, None) == -2
    assert q(FAKE, 0, 4, 8, 8, 1, FAKE2, 4, FAKE, ctypes.c_void_p(0x1010), BIG, None) == -2
    assert q(FAKE, 0, 4, 8, 8, 1, FAKE2, 4, FAKE, FAKE, 16, None) == -2
    assert q(None, 0, 0, 8, 8, 0, None, 8, FAKE, None, 0, None) == 0            # no rows: nothing to do


def test_product_and_layer_refusals():
    lib = rt.load_library()
    mm = lib.rtopk_matmul_i8
    assert mm(None, FAKE, FAKE, FAKE, None, 4, 4, 4, 4, 4, FAKE2, 0, 4, None, 0, None) == -1
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 4, 4, 4, 3, 4, FAKE2, 0, 4, None, 0, None) == -1
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 4, 4, 4, 4, 4, FAKE2, 0, 3, None, 0, None) == -1
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 4, 4, 4, 4, 4, FAKE2, 9, 4, None, 0, None) == -1
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 4, 4, 4, 4, MOST + 1, FAKE2, 0, 4, None, 0, None) == -1
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 4, 4, 140_000, 140_000, 140_000, FAKE2, 0, 4, None, 0, None) == -2
    assert mm(FAKE, FAKE, FAKE, FAKE, None, 0, 4, 4, 4, 4, FAKE2, 0, 4, None, 0, None) == 0
    fw = lib.rtopk_linear_i8
    assert fw(None, 0, 4, 8, 8, FAKE, FAKE, 4, 8, None, FAKE2, 0, 4, FAKE, BIG, None) == -1
    assert fw(FAKE, 0, 4, 8, 8, FAKE, FAKE, 4, 7, None, FAKE2, 0, 4, FAKE, BIG, None) == -1
    assert fw(FAKE, 0, 4, 8, 8, FAKE, FAKE, 4, 8, None, FAKE2, 0, 3, FAKE, BIG, None) == -1
    assert fw(FAKE, -1, 4, 8, 8, FAKE, FAKE, 4, 8, None, FAKE2, 0, 4, FAKE, BIG, None) == -1
    need = rt.linear_i8_workspace_bytes(400, 800, 400)
    assert need > 0
    assert fw(FAKE, 0, 400, 800, 800, FAKE, FAKE, 400, 800, None, FAKE2, 0, 400, None, 0, None) == -2
    assert fw(FAKE, 0, 400, 800, 800, FAKE, FAKE, 400, 800, None, FAKE2, 0, 400, FAKE, need - 1, None) == -2
    assert fw(None, 0, 0, 8, 8, None, None, 4, 8, None, None, 0, 4, None, 0, None) == 0
    bw = lib.rtopk_linear_i8_backward
    full = lambda **k: bw(*({**dict(dy=FAKE, x=FAKE, type=0, m=4, k=8, n=6, lddy=6, ldx=8, w=FAKE, s=FAKE, ldw=6, dx=FAKE2,  # noqa: E731
                                    lddx=8, dw=FAKE2, lddw=8, db=FAKE2, ws=FAKE, bytes=BIG, stream=None), **k}.values()))
    assert full(dy=None) == -1 and full(x=None) == -1 and full(w=None) == -1 and full(s=None) == -1
    assert full(type=7) == -1 and full(lddy=5) == -1 and full(ldx=7) == -1 and full(ldw=5) == -1
    assert full(lddx=7) == -1 and full(lddw=7) == -1 and full(dx=None, dw=None) == -1 and full(dw=None) == -1   # db without dw
    assert full(ws=None) == -2 and full(bytes=ctypes.c_uint64(8)) == -2


def _iterate(coefficients, steps=None, eps=1e-7, count=1, rows=4, cols=6, ldx=6, ldo=6, workspace=FAKE, size=BIG, x=FAKE, out=FAKE2,
             products=0, kind=0):
    lib = rt.load_library()
    steps = len(coefficients) // 3 if steps is None else steps
    abc = (ctypes.c_float * max(1, len(coefficients)))(*coefficients)
    xs, outs = (ctypes.c_void_p * max(1, count))(x), (ctypes.c_void_p * max(1, count))(out)
    return lib.rtopk_orthogonalize(count, xs, kind, rows, cols, ldx, steps, abc, eps, products, outs, 0, ldo, workspace, size, None)


def test_orthogonalize_refusals():
    good = list(rt.QUINTIC) * 5
    assert _iterate(good, workspace=None) == -2                  # (the arguments before it are fine)
    assert _iterate(good, size=ctypes.c_uint64(64)) == -2
    assert _iterate(good, workspace=ctypes.c_void_p(0x1010)) == -2
    for bad in (dict(count=0), dict(rows=0), dict(cols=0), dict(ldx=5), dict(ldo=5), dict(x=None), dict(out=None), dict(products=2),
                dict(kind=3), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(steps=0), dict(steps=65)):
        assert _iterate(good, workspace=None, **{k: v for k, v in bad.items()}) == -1, bad


@pytest.mark.parametrize("coefficients, fine", [
    ((1.5, -0.5, 0.0), True),                # the cubic iteration
    ((1.875, -1.25, 0.375), True),           # the quintic one that converges
    ((3.4445, -4.7750, 2.0315), True),
    ((7.0, 0.0, 0.0), False),                # the second step starts at 7 and leaves for 49
    ((0.0, 0.0, 0.0), True),
    ((8.0, -8.0, 0.0), False),               # largest between the ends: 8 s - 8 s^3 at s = 3^-1/2 is 3.08, at 3.08 it is far out
    ((math.nan, 0.0, 0.0), False),
    ((1.0, math.inf, 0.0), False),
])
def test_coefficients_whose_iterates_leave_the_range_are_refused(coefficients, fine):
    assert _iterate(list(coefficients) * 5, workspace=None) == (-2 if fine else -1)


def test_one_step_may_take_what_five_may_not():
    assert _iterate([7.0, 0.0, 0.0], workspace=None) == -2
    assert _iterate([7.6, 0.0, 0.0], workspace=None) == -1
    assert _iterate([0.0, 70.0, -70.0], workspace=None) == -1     # s: 70 (s^3 - s^5) stays under 13.02, over 7.5
    assert _iterate([60.0, -120.0, 62.0], workspace=None) == -1


def test_master_step_refusals():
    lib = rt.load_library()
    abc = (ctypes.c_float * 15)(*(list(rt.QUINTIC) * 5))
    one = lambda p: (ctypes.c_void_p * 1)(p)     # noqa: E731

    def call(idx=0x1000, val=0x2000, n=2, k=3, rows=4, cols=6, omega=0x100000, velocity=0x200000, ws=FAKE, size=BIG, count=1):
        return lib.rtopk_aggregate_update_orthogonal(count, one(idx), one(val), n, k, rows, cols, 0.1, 1.0, 0.9, 1, 0.0, 1.0, 5, abc,
                                                     1e-7, 0, one(omega), one(velocity), ws, size, None)

    assert call(ws=None) == -2 and call(size=ctypes.c_uint64(8)) == -2
    assert call(idx=None) == -1 and call(val=None) == -1 and call(omega=None) == -1 and call(velocity=None) == -1
    assert call(n=0) == -1 and call(k=0) == -1 and call(rows=0) == -1 and call(count=0) == -1
    assert call(velocity=0x100000 + 4 * 23) == -1                # the last element of omega


def test_binding_refuses_tensors_that_are_not_matrices_on_the_gpu():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    for call in (lambda: rt.orthogonalize([x], [x]), lambda: rt.quantize_i8(x, x, x),
                 lambda: rt.linear_i8(x, x, x, x), lambda: rt.matmul_i8(x, x, x, x, x)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        rt.orthogonalize([], [])
    with pytest.raises(ValueError):
        rt.linear_i8_backward(x, x, x, x, None, None)
