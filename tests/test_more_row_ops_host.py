"""CPU tests of the argument checks of mgn_quant4, mgn_dequant4, mgn_matmul4,
mgn_group_norm_* and mgn_grad_*: every refusal comes before any device work, so
the pointers here are made up and never followed; workspace sizes; the pieces of
a list of gradients, which are made on the host."""
import ctypes as C

import pytest

from paper_2304_00338_amd import mgn

P = 0x7000000000  # a 16-byte aligned address that nothing reads
NONE = None


def L():
    return mgn.lib()


def quant4(x=P, xt=0, rows=4, cols=130, ldx=130, q=P, ldq=80, s=P, qt=P + 4096, ldqt=16, st=P + 8192, cs=NONE, acc=0, ws=NONE, n=0):
    return L().mgn_quant4(x, xt, rows, cols, ldx, q, ldq, s, qt, ldqt, st, cs, acc, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=NONE), mgn.ERR_ARG), (dict(xt=2), mgn.ERR_ARG), (dict(rows=-1), mgn.ERR_ARG), (dict(cols=-1), mgn.ERR_ARG),
    (dict(rows=1 << 31), mgn.ERR_SHAPE), (dict(cols=1 << 31), mgn.ERR_SHAPE), (dict(ldx=129), mgn.ERR_ARG),
    (dict(x=P + 2), mgn.ERR_ARG), (dict(x=P + 1, xt=1), mgn.ERR_ARG), (dict(s=NONE), mgn.ERR_ARG),
    (dict(q=NONE), mgn.ERR_ARG), (dict(st=NONE), mgn.ERR_ARG), (dict(ldq=64), mgn.ERR_ARG), (dict(ldq=88), mgn.ERR_ARG),
    (dict(q=P + 8), mgn.ERR_ARG), (dict(ldqt=0), mgn.ERR_ARG), (dict(qt=P + 4), mgn.ERR_ARG), (dict(s=P + 2), mgn.ERR_ARG),
    (dict(rows=1 << 30, cols=1 << 30, ldx=1 << 30, ldq=1 << 29, ldqt=1 << 29), mgn.ERR_SHAPE),
    (dict(cs=P), mgn.ERR_WORKSPACE), (dict(cs=P, ws=P, n=519), mgn.ERR_WORKSPACE),
    (dict(cs=P, ws=P + 4, n=520), mgn.ERR_WORKSPACE), (dict(cs=P + 2, ws=P, n=520), mgn.ERR_ARG),
    (dict(ldx=1 << 59), mgn.ERR_ARG), (dict(q=P + 4096, qt=P + 4096), mgn.ERR_ARG), (dict(st=P, s=P, q=P + 64), mgn.ERR_ARG),
])
def test_quant4_refusals(kw, code):
    assert quant4(**kw) == code
    assert mgn.last_error().startswith("mgn_quant4")


def test_quant4_empty():
    assert quant4(cols=0) == mgn.OK
    assert quant4(q=NONE, s=NONE, qt=NONE, st=NONE) == mgn.OK
    n = C.c_size_t()
    assert L().mgn_quant4_workspace(300, 1000, C.byref(n)) == mgn.OK and n.value == 3 * 1000 * 4
    assert L().mgn_quant4_workspace(-1, 1, C.byref(n)) == mgn.ERR_ARG
    assert L().mgn_quant4_workspace(1, 1, None) == mgn.ERR_ARG


def mat4(q=P, scale=P, rows=40, cols=130, ld=80):
    return mgn.CMat4(q, scale, rows, cols, ld)


MATS = [
    (dict(q=NONE), mgn.ERR_ARG), (dict(scale=NONE), mgn.ERR_ARG), (dict(q=P + 8), mgn.ERR_ARG),
    (dict(scale=P + 2), mgn.ERR_ARG), (dict(ld=64), mgn.ERR_ARG), (dict(ld=81), mgn.ERR_ARG), (dict(rows=-1), mgn.ERR_ARG),
    (dict(rows=1 << 31), mgn.ERR_SHAPE), (dict(cols=-1), mgn.ERR_ARG), (dict(cols=1 << 31, ld=1 << 30), mgn.ERR_SHAPE),
    (dict(ld=1 << 60), mgn.ERR_ARG),
]


@pytest.mark.parametrize("kw,code", MATS)
def test_mat4_refusals(kw, code):
    good, bad = mat4(), mat4(**kw)
    assert L().mgn_dequant4(C.byref(bad), 0, P, 1 << 20, None) == code
    for a, b in ((good, bad), (bad, good)):
        assert L().mgn_matmul4(C.byref(a), C.byref(b), None, 0, P, 1 << 20, NONE, 0, None) == code


def test_dequant4_refusals():
    a = mat4()
    assert L().mgn_dequant4(None, 0, P, 130, None) == mgn.ERR_ARG
    for yt, y, ld in ((2, P, 130), (0, NONE, 130), (0, P + 2, 130), (1, P + 1, 130), (0, P, 129), (0, P, 1 << 58)):
        assert L().mgn_dequant4(C.byref(a), yt, y, ld, None) == mgn.ERR_ARG
    assert L().mgn_dequant4(C.byref(mat4(rows=0)), 0, NONE, 0, None) == mgn.OK
    assert L().mgn_dequant4(C.byref(mat4(cols=0)), 0, NONE, 0, None) == mgn.OK


def test_matmul4_refusals():
    a, b = mat4(), mat4(rows=50)

    def go(x=a, y=b, ep=None, ct=0, c=P, ldc=50, ws=NONE, n=0):
        return L().mgn_matmul4(C.byref(x), C.byref(y), None if ep is None else C.byref(ep), ct, c, ldc, ws, n, None)
    assert go(y=mat4(cols=131)) == mgn.ERR_SHAPE
    for kw in (dict(ct=2), dict(c=NONE), dict(c=P + 2), dict(ldc=49), dict(ldc=1 << 59)):
        assert go(**kw) == mgn.ERR_ARG
    E = mgn.Epilogue
    for ep in (E(act=3), E(act=-1), E(bias=P + 2), E(act=2), E(act=2, aux=P, aux_type=2, ldaux=50),
               E(act=2, aux=P, aux_type=0, ldaux=49), E(act=2, aux=P + 2, aux_type=0, ldaux=50)):
        assert go(ep=ep) == mgn.ERR_ARG
    assert L().mgn_matmul4(None, C.byref(b), None, 0, P, 50, NONE, 0, None) == mgn.ERR_ARG
    big = mat4(rows=(1 << 31) - 1, cols=32, ld=16)
    assert go(x=big, y=mat4(rows=1 << 20, cols=32, ld=16), ldc=1 << 20) == mgn.ERR_SHAPE
    assert go(x=mat4(rows=3, cols=32, ld=16), y=big, ldc=1 << 31) == mgn.ERR_SHAPE  # few rows may be tiles too
    # rows 2^28 bytes apart
    assert go(x=mat4(ld=1 << 28)) == mgn.ERR_ARG and go(y=mat4(rows=50, ld=1 << 28)) == mgn.ERR_ARG
    assert go(x=mat4(rows=0)) == mgn.OK and go(y=mat4(rows=0)) == mgn.OK
    n = C.c_size_t()
    assert L().mgn_matmul4_workspace(128, 256, 852640, C.byref(n)) == mgn.OK and n.value > 0
    deep = [mat4(rows=128, cols=852640, ld=426320), mat4(rows=256, cols=852640, ld=426320)]
    assert go(x=deep[0], y=deep[1], ldc=256, ws=P, n=n.value - 1) == mgn.ERR_WORKSPACE
    assert go(x=deep[0], y=deep[1], ldc=256, ws=P + 8, n=n.value) == mgn.ERR_WORKSPACE
    assert L().mgn_matmul4_workspace(-1, 1, 1, C.byref(n)) == mgn.ERR_ARG
    assert L().mgn_matmul4_workspace(1 << 31, 1, 1, C.byref(n)) == mgn.ERR_SHAPE


def gn(rows=64, cols=96, groups=32, type=0, act=3, eps=1e-5, gamma=P, beta=P, ptr=NONE, n=4):
    return mgn.CGroupNorm(rows, cols, groups, type, act, eps, gamma, beta, ptr, n)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), mgn.ERR_ARG), (dict(rows=1 << 31), mgn.ERR_SHAPE), (dict(cols=0, groups=1), mgn.ERR_SHAPE),
    (dict(cols=16385, groups=1), mgn.ERR_SHAPE), (dict(groups=0), mgn.ERR_ARG), (dict(groups=31), mgn.ERR_ARG),
    (dict(groups=192), mgn.ERR_ARG), (dict(type=2), mgn.ERR_ARG), (dict(act=2), mgn.ERR_ARG), (dict(act=4), mgn.ERR_ARG),
    (dict(eps=0.0), mgn.ERR_ARG), (dict(eps=float("nan")), mgn.ERR_ARG), (dict(eps=float("inf")), mgn.ERR_ARG),
    (dict(gamma=P + 2), mgn.ERR_ARG), (dict(beta=P + 1), mgn.ERR_ARG), (dict(ptr=P + 2), mgn.ERR_ARG),
    (dict(n=-1), mgn.ERR_ARG), (dict(n=3), mgn.ERR_ARG), (dict(n=0), mgn.ERR_ARG),
    (dict(n=(1 << 21) + 1, ptr=P), mgn.ERR_SHAPE),
])
def test_group_norm_refusals(kw, code):
    op, r, n = gn(**kw), mgn.Rows(P, 96), C.c_size_t()
    ws, big = P, 1 << 50
    assert L().mgn_group_norm_workspace(C.byref(op), 0, C.byref(n)) == code
    assert L().mgn_group_norm_forward(C.byref(op), r, r, P, ws, big, None) == code
    assert L().mgn_group_norm_backward(C.byref(op), r, P, r, r, P, P + 4096, 0, ws, big, None) == code


def test_group_norm_buffers():
    op, big = gn(rows=100000, n=4), 1 << 50
    good = mgn.Rows(P, 96)
    bad = [mgn.Rows(None, 96), mgn.Rows(P, 95), mgn.Rows(P + 2, 96), mgn.Rows(P, 1 << 59)]
    for b in bad:
        assert L().mgn_group_norm_forward(C.byref(op), b, good, P, P, big, None) == mgn.ERR_ARG
        assert L().mgn_group_norm_forward(C.byref(op), good, b, P, P, big, None) == mgn.ERR_ARG
        for i in range(3):
            r = [good] * 3
            r[i] = b
            assert L().mgn_group_norm_backward(C.byref(op), r[0], P, r[1], r[2], P, NONE, 0, P, big, None) == mgn.ERR_ARG
    # in place of another layout
    assert L().mgn_group_norm_forward(C.byref(op), good, mgn.Rows(P, 128), P, P, big, None) == mgn.ERR_ARG
    assert L().mgn_group_norm_backward(C.byref(op), good, P, mgn.Rows(P + 4096, 100), mgn.Rows(P + 4096, 96), NONE, NONE, 0,
                                       P, big, None) == mgn.ERR_ARG
    other = mgn.Rows(P + 4096, 96)
    assert L().mgn_group_norm_forward(C.byref(op), good, other, P + 4, P, big, None) == mgn.ERR_ARG
    assert L().mgn_group_norm_backward(C.byref(op), good, None, other, other, P, NONE, 0, P, big, None) == mgn.ERR_ARG
    assert L().mgn_group_norm_backward(C.byref(op), good, P, other, other, P, P, 0, P, big, None) == mgn.ERR_ARG
    assert L().mgn_group_norm_backward(C.byref(op), good, P, other, other, P + 2, NONE, 0, P, big, None) == mgn.ERR_ARG
    for back in (0, 1):
        n = C.c_size_t()
        assert L().mgn_group_norm_workspace(C.byref(op), back, C.byref(n)) == mgn.OK and n.value > 0
        for ws, size in ((NONE, n.value), (P, n.value - 1), (P + 8, n.value)):
            if back:
                rc = L().mgn_group_norm_backward(C.byref(op), good, P, other, other, P, NONE, 0, ws, size, None)
            else:
                rc = L().mgn_group_norm_forward(C.byref(op), good, other, P, ws, size, None)
            assert rc == mgn.ERR_WORKSPACE
    assert L().mgn_group_norm_workspace(C.byref(op), 0, None) == mgn.ERR_ARG
    assert L().mgn_group_norm_workspace(None, 0, C.byref(n)) == mgn.ERR_ARG
    none = gn(rows=0, n=0)
    assert L().mgn_group_norm_forward(C.byref(none), mgn.Rows(None, 0), mgn.Rows(None, 0), None, None, 0, None) == mgn.OK


def pieces(*tensors, fill=True):
    t = (mgn.CTensor * max(len(tensors), 1))(*[mgn.CTensor(*x) for x in tensors])
    n = C.c_int64(-7)
    rc = L().mgn_grad_pieces(t, len(tensors), None, C.byref(n))
    if rc != mgn.OK:
        assert n.value == -7
        return rc
    p = (mgn.CPiece * max(n.value, 1))()
    assert L().mgn_grad_pieces(t, len(tensors), p, C.byref(n)) == mgn.OK
    return [(x.data, x.out, x.n, x.types) for x in p[:n.value]]


def test_pieces():
    size = L().mgn_grad_piece()
    big = 2 * size + 5
    got = pieces((P, P, big, 0, 0), (P + 4 * big, P + (1 << 30), 3, 1, 0), (None, None, 0, 0, 0), (P + (1 << 31), None, size, 1, 0))
    assert got == [(P, P, size, 0), (P + 4 * size, P + 4 * size, size, 0), (P + 8 * size, P + 8 * size, 5, 0),
                   (P + 4 * big, P + (1 << 30), 3, 1), (P + (1 << 31), None, size, 1)]
    assert pieces() == []
    # the same gradient twice, into two places; neighbours without a gap
    assert len(pieces((P, P + 4096, 64, 0, 0), (P, P + 4352, 64, 0, 0))) == 2
    assert len(pieces((P, P + 4096, 64, 0, 1), (P + 256, P + 4224, 64, 0, 1))) == 2


@pytest.mark.parametrize("tensors", [
    [(P, P, -1, 0, 0)], [(None, P, 4, 0, 0)], [(P + 2, P, 4, 0, 0)], [(P, P + 2, 4, 0, 0)], [(P, P, 4, 2, 0)],
    [(P, P, 4, 0, 2)], [(P, P, 4, 0, 1)], [(P, P + 4, 4, 0, 0)],
    [(P, P, 64, 0, 0), (P, P, 64, 0, 0)],                       # in place twice
    [(P, P + 4096, 64, 0, 0), (P + 1024, P + 4348, 64, 0, 0)],  # places overlap
    [(P, P + 1024, 64, 0, 0), (P + 1024, P + 4096, 64, 0, 0)],  # a place is another's gradient
    [(P, P, 64, 0, 0), (P + 252, P + 4096, 4, 0, 0)],
    [(P, P + 4096, 4096, 0, 0), (P + 64, P + 32768, 8, 0, 0), (P + 65536, P + 1024, 8, 0, 0)],
    [(P, P, 1 << 60, 0, 0)],
])
def test_pieces_refusals(tensors):
    assert pieces(*tensors) == mgn.ERR_ARG
    assert mgn.last_error().startswith("mgn_grad_pieces")


def test_clip_refusals():
    n = C.c_size_t()
    assert L().mgn_grad_norm_workspace(5, C.byref(n)) == mgn.OK and n.value == 40
    assert L().mgn_grad_norm_workspace(-1, C.byref(n)) == mgn.ERR_ARG
    assert L().mgn_grad_norm_workspace(1, None) == mgn.ERR_ARG

    def clip(p=P, k=5, most=1.0, norm=P, given=0, ws=P, size=40):
        return L().mgn_grad_clip(p, k, most, norm, given, ws, size, None)
    for kw in (dict(p=None), dict(p=P + 4), dict(k=-1), dict(k=1 << 31), dict(most=-1.0), dict(most=float("nan")),
               dict(norm=None), dict(norm=P + 2)):
        assert clip(**kw) == mgn.ERR_ARG
    for kw in (dict(ws=None), dict(size=39), dict(ws=P + 8)):
        assert clip(**kw) == mgn.ERR_WORKSPACE
    assert L().mgn_grad_norm(P, 5, None, P, 40, None) == mgn.ERR_ARG
    assert L().mgn_grad_norm(P, 5, P, P, 39, None) == mgn.ERR_WORKSPACE
    assert L().mgn_grad_pieces(None, 1, None, C.byref(C.c_int64())) == mgn.ERR_ARG
    assert L().mgn_grad_pieces(None, 0, None, None) == mgn.ERR_ARG
