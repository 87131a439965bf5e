"""CPU tests of the row operators' argument checks (mgn_quant8, mgn_matmul8,
mgn_norm_gate_*): every refusal comes before any device work, so the pointers
here are made up and never followed; workspace sizes; empty calls."""
import ctypes as C

import pytest

from paper_2304_00338_amd import mgn

P = 0x7000000000  # a 16-byte aligned address that nothing reads
NONE = None


def L():
    return mgn.lib()


def quant8(x=P, xt=0, rows=4, cols=130, ldx=130, fmt=mgn.E4M3, block=1, q=P, ldq=144, s=P, qt=P, ldqt=16, st=P, cs=NONE,
           acc=0, ws=NONE, n=0):
    return L().mgn_quant8(x, xt, rows, cols, ldx, fmt, block, q, ldq, s, qt, ldqt, st, cs, acc, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=NONE), mgn.ERR_ARG), (dict(xt=2), mgn.ERR_ARG), (dict(xt=-1), mgn.ERR_ARG), (dict(rows=-1), mgn.ERR_ARG),
    (dict(cols=-1), mgn.ERR_ARG), (dict(rows=1 << 31), mgn.ERR_SHAPE), (dict(cols=1 << 31), mgn.ERR_SHAPE),
    (dict(ldx=129), mgn.ERR_ARG), (dict(x=P + 2), mgn.ERR_ARG), (dict(x=P + 1, xt=1), mgn.ERR_ARG),
    (dict(fmt=1), mgn.ERR_ARG), (dict(block=2), mgn.ERR_ARG), (dict(block=64), mgn.ERR_ARG), (dict(s=NONE), mgn.ERR_ARG),
    (dict(q=NONE), mgn.ERR_ARG), (dict(st=NONE), mgn.ERR_ARG), (dict(ldq=143), mgn.ERR_ARG), (dict(ldq=128), mgn.ERR_ARG),
    (dict(ldq=136), mgn.ERR_ARG), (dict(q=P + 8), mgn.ERR_ARG), (dict(ldqt=0), mgn.ERR_ARG), (dict(qt=P + 4), mgn.ERR_ARG),
    (dict(rows=1 << 30, cols=1 << 30, ldx=1 << 30, ldq=1 << 30, ldqt=1 << 30), mgn.ERR_SHAPE),
    (dict(cs=P), mgn.ERR_WORKSPACE), (dict(cs=P, ws=P, n=519), mgn.ERR_WORKSPACE),
    (dict(cs=P, ws=P + 4, n=520), mgn.ERR_WORKSPACE), (dict(cs=P + 2, ws=P, n=520), mgn.ERR_ARG),
])
def test_quant8_refusals(kw, code):
    assert quant8(**kw) == code
    assert mgn.last_error().startswith("mgn_quant8")


def test_quant8_empty():
    assert quant8(cols=0) == mgn.OK
    assert quant8(q=NONE, s=NONE, qt=NONE, st=NONE) == mgn.OK
    n = C.c_size_t()
    assert L().mgn_quant8_workspace(129, 5, C.byref(n)) == mgn.OK and n.value == 2 * 5 * 4
    assert L().mgn_quant8_workspace(129, 5, None) == mgn.ERR_ARG


def mat8(q=P, scale=P, rows=3, cols=130, ld=144, fmt=mgn.E4M3, block=1):
    return mgn.CMat8(q, scale, rows, cols, ld, fmt, block)


def matmul8(a=None, b=None, ep=None, ct=0, c=P, ldc=5, ws=NONE, n=0):
    a, b = a or mat8(), b or mat8(rows=5)
    return L().mgn_matmul8(C.byref(a), C.byref(b), C.byref(ep) if ep else None, ct, c, ldc, ws, n, None)


def ep(bias=NONE, act=0, aux_type=0, aux=NONE, ldaux=0, acc=0):
    return mgn.Epilogue(bias, act, aux_type, aux, ldaux, acc)


@pytest.mark.parametrize("kw,code", [
    (dict(a=mat8(q=NONE)), mgn.ERR_ARG), (dict(a=mat8(scale=NONE)), mgn.ERR_ARG), (dict(a=mat8(q=P + 8)), mgn.ERR_ARG),
    (dict(a=mat8(scale=P + 2)), mgn.ERR_ARG), (dict(a=mat8(ld=130)), mgn.ERR_ARG), (dict(a=mat8(ld=128)), mgn.ERR_ARG),
    (dict(a=mat8(fmt=0)), mgn.ERR_ARG), (dict(a=mat8(block=32)), mgn.ERR_ARG), (dict(a=mat8(rows=-1)), mgn.ERR_ARG),
    (dict(a=mat8(rows=1 << 31)), mgn.ERR_SHAPE), (dict(b=mat8(cols=131)), mgn.ERR_SHAPE),
    (dict(a=mat8(rows=1 << 30), b=mat8(rows=1 << 30), ldc=1 << 30), mgn.ERR_SHAPE),
    (dict(b=mat8(q=NONE)), mgn.ERR_ARG), (dict(ct=2), mgn.ERR_ARG), (dict(c=NONE), mgn.ERR_ARG), (dict(ldc=4), mgn.ERR_ARG),
    (dict(c=P + 2), mgn.ERR_ARG), (dict(ep=ep(act=3)), mgn.ERR_ARG), (dict(ep=ep(act=-1)), mgn.ERR_ARG),
    (dict(ep=ep(bias=P + 2)), mgn.ERR_ARG), (dict(ep=ep(act=2)), mgn.ERR_ARG),
    (dict(ep=ep(act=2, aux=P, ldaux=4)), mgn.ERR_ARG), (dict(ep=ep(act=2, aux=P, ldaux=5, aux_type=3)), mgn.ERR_ARG),
    (dict(ep=ep(act=2, aux=P + 2, ldaux=5)), mgn.ERR_ARG),
])
def test_matmul8_refusals(kw, code):
    assert matmul8(**kw) == code
    assert mgn.last_error().startswith("mgn_matmul8")


def test_matmul8_null_and_empty():
    a = mat8()
    assert L().mgn_matmul8(None, C.byref(a), None, 0, P, 5, None, 0, None) == mgn.ERR_ARG
    assert L().mgn_matmul8(C.byref(a), None, None, 0, P, 5, None, 0, None) == mgn.ERR_ARG
    assert matmul8(a=mat8(rows=0, q=NONE, scale=NONE), c=NONE) == mgn.OK
    assert matmul8(b=mat8(rows=0, q=NONE, scale=NONE), c=NONE) == mgn.OK
    n = C.c_size_t()
    assert L().mgn_matmul8_workspace(-1, 5, 5, C.byref(n)) == mgn.ERR_ARG
    assert L().mgn_matmul8_workspace(1 << 31, 5, 5, C.byref(n)) == mgn.ERR_SHAPE
    # long sums of a small result are split: that takes a workspace
    assert L().mgn_matmul8_workspace(16, 128, 1 << 20, C.byref(n)) == mgn.OK
    if n.value:
        big = dict(cols=1 << 20, ld=1 << 20)
        assert matmul8(a=mat8(rows=16, **big), b=mat8(rows=128, **big), ldc=128) == mgn.ERR_WORKSPACE
        assert matmul8(a=mat8(rows=16, **big), b=mat8(rows=128, **big), ldc=128, ws=P, n=n.value - 1) == mgn.ERR_WORKSPACE


def op(rows=3, cols=7, xt=0, bt=1, post=1, pre=2, eps=1e-5, gate=NONE, ptr=NONE, gates=0):
    return mgn.CNormGate(rows, cols, xt, bt, post, pre, eps, 1.0, 1.0, NONE, NONE, NONE, NONE, gate, ptr, gates)


def R(p=P, ld=7):
    return mgn.Rows(p, ld)


def forward(o=None, x=R(), b=R(), y=R(), z=R(), stats=NONE):
    return L().mgn_norm_gate_forward(C.byref(o or op()), x, b, y, z, stats, None)


def backward(o=None, x=R(), b=R(), stats=P, dy=R(), dz=R(), dx=R(), db=R(), grads=None, ws=P, n=1 << 40):
    return L().mgn_norm_gate_backward(C.byref(o or op()), x, b, stats, dy, dz, dx, db,
                                      C.byref(grads) if grads else None, ws, n, None)


BAD_OPS = [
    (op(rows=-1), mgn.ERR_ARG), (op(rows=1 << 31), mgn.ERR_SHAPE), (op(cols=0), mgn.ERR_SHAPE),
    (op(cols=mgn.NORM_MAX_COLS + 1), mgn.ERR_SHAPE), (op(xt=2), mgn.ERR_ARG), (op(bt=-1), mgn.ERR_ARG),
    (op(post=3), mgn.ERR_ARG), (op(pre=-1), mgn.ERR_ARG), (op(eps=0.0), mgn.ERR_ARG), (op(eps=-1.0), mgn.ERR_ARG),
    (op(eps=float("nan")), mgn.ERR_ARG), (op(eps=float("inf")), mgn.ERR_ARG), (op(gates=1), mgn.ERR_ARG),
    (op(gates=2, gate=P), mgn.ERR_ARG), (op(ptr=P), mgn.ERR_ARG), (op(gates=-1, gate=P), mgn.ERR_ARG),
]


@pytest.mark.parametrize("o,code", BAD_OPS)
def test_norm_gate_bad_op(o, code):
    assert forward(o) == code
    assert backward(o) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=R(NONE)), mgn.ERR_ARG), (dict(b=R(NONE)), mgn.ERR_ARG), (dict(y=R(NONE)), mgn.ERR_ARG),
    (dict(z=R(NONE)), mgn.ERR_ARG), (dict(x=R(ld=6)), mgn.ERR_ARG), (dict(x=R(P + 2)), mgn.ERR_ARG),
    (dict(b=R(P + 1)), mgn.ERR_ARG), (dict(stats=P + 8), mgn.ERR_ARG),
])
def test_norm_gate_forward_refusals(kw, code):
    assert forward(**kw) == code
    assert mgn.last_error().startswith("mgn_norm_gate_forward")


@pytest.mark.parametrize("kw,code", [
    (dict(x=R(NONE)), mgn.ERR_ARG), (dict(b=R(NONE)), mgn.ERR_ARG), (dict(dx=R(NONE)), mgn.ERR_ARG),
    (dict(db=R(NONE)), mgn.ERR_ARG), (dict(stats=NONE), mgn.ERR_ARG), (dict(stats=P + 4), mgn.ERR_ARG),
    (dict(dy=R(ld=6)), mgn.ERR_ARG), (dict(dz=R(ld=6)), mgn.ERR_ARG), (dict(o=op(pre=0)), mgn.ERR_ARG),
    (dict(ws=NONE), mgn.ERR_WORKSPACE), (dict(ws=P + 8), mgn.ERR_WORKSPACE), (dict(n=3), mgn.ERR_WORKSPACE),
    (dict(grads=mgn.CNormGateGrads(P + 2, NONE, NONE, NONE, NONE, 0)), mgn.ERR_ARG),
])
def test_norm_gate_backward_refusals(kw, code):
    assert backward(**kw) == code
    assert mgn.last_error().startswith("mgn_norm_gate_backward")


def test_norm_gate_null_and_empty():
    assert L().mgn_norm_gate_forward(None, R(), R(), R(), R(), None, None) == mgn.ERR_ARG
    assert forward(op(rows=0), x=R(NONE), b=R(NONE), y=R(NONE), z=R(NONE)) == mgn.OK
    n = C.c_size_t()
    assert L().mgn_norm_gate_workspace(0, 7, C.byref(n)) == mgn.OK and n.value == 0
    assert L().mgn_norm_gate_workspace(5, 0, C.byref(n)) == mgn.ERR_SHAPE
    assert L().mgn_norm_gate_workspace(-5, 4, C.byref(n)) == mgn.ERR_ARG
    assert backward(op(rows=0), x=R(NONE), b=R(NONE), stats=NONE, dx=R(NONE), db=R(NONE), ws=NONE, n=0) == mgn.OK


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(4, 8)
    for call in (lambda: mgn.mgn_quant8(x), lambda: mgn.Mat8(x.to(torch.float8_e4m3fn), x),
                 lambda: mgn.mgn_matmul8(x, x), lambda: mgn.mgn_norm_gate_forward(x, x)):
        with pytest.raises(mgn.MgnError) as e:
            call()
        assert e.value.code == mgn.ERR_ARG


def test_matmul8_tiles_of_a_grid():
    """2^24 tiles of 128 x 128 are refused, rows of b beside few rows of a are not tiles."""
    tall = dict(cols=16, ld=16)
    assert matmul8(a=mat8(rows=(1 << 31) - 1, **tall), b=mat8(rows=1, **tall), ldc=1) == mgn.ERR_SHAPE
    assert "too large" in mgn.last_error()


Q = P + (1 << 20)


@pytest.mark.parametrize("kw", [
    dict(x=R(ld=8), y=R(), z=R(Q), b=R(Q)), dict(x=R(), y=R(), b=R(Q), z=R(Q, 8)),  # in place, ld differs
    dict(x=R(), b=R(Q), y=R(), z=R()),  # y and z the same
])
def test_norm_gate_forward_in_place_refusals(kw):
    assert forward(**kw) == mgn.ERR_ARG
    assert "in place" in mgn.last_error() or "same" in mgn.last_error()


@pytest.mark.parametrize("kw", [
    dict(x=R(ld=8), dx=R(), db=R(Q)), dict(dy=R(ld=8), dx=R(), db=R(Q)), dict(b=R(Q, 8), dx=R(), db=R(Q)),
    dict(dz=R(Q, 8), b=R(Q), dx=R(), db=R(Q)), dict(dx=R(), db=R()),
])
def test_norm_gate_backward_in_place_refusals(kw):
    assert backward(**kw) == mgn.ERR_ARG
    assert "in place" in mgn.last_error() or "same" in mgn.last_error()


def test_far_rows_refused():
    far = 1 << 59  # 4 rows of it end past 63 bits of bytes
    assert quant8(ldx=far) == mgn.ERR_ARG and quant8(ldq=far) == mgn.ERR_ARG
    assert matmul8(a=mat8(ld=far)) == mgn.ERR_ARG and matmul8(ldc=far) == mgn.ERR_ARG
    assert forward(x=R(ld=far)) == mgn.ERR_ARG
