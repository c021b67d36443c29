"""Arguments that the calls around the products refuse, before anything is enqueued (no GPU needed: the addresses are never read)."""
import ctypes as C
import os

import pytest

FAKE = 1 << 30
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -5
NAN = float("nan")


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    m.lib()
    return m


def _ref(x):
    return C.byref(x) if x is not None else None


BAD_MASKS = [dict(p=-0.1), dict(p=1.0), dict(p=NAN), dict(p=1 - 2.0 ** -18), dict(step=FAKE + 4)]


def _mask(metis, p=0.1, seed=1, step=None):
    return metis.Mask(p, seed, step)


def test_dropout(metis):
    L = metis.lib()

    def call(x=(4, 40, 40, 0), y=(4, 40, 40, 0), res=None, xp=FAKE, yp=FAKE, mask={}):
        a, o, r = metis.Mat(xp, *x), metis.Mat(yp, *y), metis.Mat(FAKE, *res) if res else None
        m = _mask(metis, **mask) if mask is not None else None
        return L.metis_dropout(None, C.byref(a), _ref(m), _ref(r), C.byref(o))

    assert call(x=(0, 40, 40, 0), y=(0, 40, 40, 0)) == 0
    assert call(xp=None) == INVALID and call(yp=None) == INVALID and call(mask=None) == INVALID
    for m in BAD_MASKS:
        assert call(mask=m) == INVALID, m
    assert call(x=(4, 40, 40, 2)) == INVALID and call(x=(4, 40, 40, 1)) == INVALID and call(res=(4, 40, 40, 1)) == INVALID
    assert call(x=(5, 40, 40, 0)) == SHAPE and call(x=(4, 41, 41, 0)) == SHAPE and call(y=(4, 40, 39, 0)) == SHAPE and call(res=(4, 40, 39, 0)) == SHAPE
    assert call(x=(4, 0, 0, 0), y=(4, 0, 0, 0)) == SHAPE
    huge = (1 << 29) + 8
    assert call(x=(4, huge, huge, 0), y=(4, huge, huge, 0)) == UNSUPPORTED
    assert call(x=(1 << 33, 8, 8, 0), y=(1 << 33, 8, 8, 0)) == UNSUPPORTED
    assert L.metis_dropout(None, None, None, None, None) == INVALID


def test_linear(metis):
    L = metis.lib()

    def call(x=(4, 64, 64, 0), xq=None, w=(40, 64), y=(4, 40, 40, 0), pre=None, res=None, act=0, mask=None, bias=None, xp=FAKE, wp=FAKE, yp=FAKE, ws=FAKE,
             size=1 << 40, codes=FAKE, scales=FAKE):
        X, Q = metis.Mat(xp, *x) if x else None, metis.MxFp4(codes, scales, *xq) if xq else None
        W, Y = metis.MxFp4(wp, FAKE, *w), metis.Mat(yp, *y)
        p, r, m = metis.Mat(FAKE, *pre) if pre else None, metis.Mat(FAKE, *res) if res else None, _mask(metis, **mask) if mask is not None else None
        ptr = lambda v: C.pointer(v) if v is not None else None
        e = metis.Epilogue(bias, act, ptr(p), ptr(m), ptr(r))
        return L.metis_mxfp4_linear(None, _ref(X), _ref(Q), C.byref(W), C.byref(e), C.byref(Y), ws, size)

    assert call(x=(0, 64, 64, 0), y=(0, 40, 40, 0)) == 0 and call(x=None, xq=(0, 64), y=(0, 40, 40, 0)) == 0
    assert call(x=None) == INVALID and call(xq=(4, 64)) == INVALID                       # neither, both
    assert call(xp=None) == INVALID and call(wp=None) == INVALID and call(yp=None) == INVALID and call(x=None, xq=(4, 64), codes=None) == INVALID
    assert call(act=5) == INVALID and call(act=-1) == INVALID and call(bias=FAKE + 2) == INVALID
    for m in BAD_MASKS:
        assert call(mask=m) == INVALID, m
    assert call(x=(4, 64, 64, 7)) == INVALID and call(y=(4, 40, 40, 7)) == INVALID and call(pre=(4, 40, 40, 1)) == INVALID and call(res=(4, 40, 40, 1)) == INVALID
    assert call(w=(40, 48), x=(4, 48, 48, 0)) == INVALID and call(w=(40, 32)) == SHAPE and call(x=(4, 64, 63, 0)) == SHAPE and call(x=(4, 64, 68, 0)) == SHAPE
    assert call(xp=FAKE + 8) == SHAPE and call(wp=FAKE + 8) == SHAPE and call(x=None, xq=(4, 64), codes=FAKE + 8) == SHAPE
    assert call(y=(5, 40, 40, 0)) == SHAPE and call(y=(4, 41, 41, 0)) == SHAPE and call(y=(4, 40, 39, 0)) == SHAPE
    assert call(pre=(4, 41, 41, 0)) == SHAPE and call(pre=(4, 40, 39, 0)) == SHAPE and call(res=(5, 40, 40, 0)) == SHAPE
    need, many = L.metis_mxfp4_linear_workspace_bytes(20, 40, 64), dict(x=(20, 64, 64, 0), y=(20, 40, 40, 0))
    assert need >= 20 * 32 + 20 * 2 and call(size=need - 1, **many) == WORKSPACE and call(ws=None, **many) == WORKSPACE
    assert call(ws=FAKE + 16, **many) == INVALID and L.metis_mxfp4_linear_workspace_bytes(4, 40, 64) == 0
    assert L.metis_mxfp4_linear_workspace_bytes(4, 40, 48) == 0 and L.metis_mxfp4_linear_workspace_bytes(0, 40, 64) == 0
    big = 1 << 28
    assert call(x=(4, 64, 64, 0), w=(big, 64), y=(4, big, big, 0)) == UNSUPPORTED
    assert call(x=(big, 64, 64, 0), y=(big, 40, 40, 0)) == UNSUPPORTED and call(x=None, xq=(big, 64), y=(big, 40, 40, 0)) == UNSUPPORTED
    assert L.metis_mxfp4_linear(None, None, None, None, None, None, None, 0) == INVALID


def test_linear_grads(metis):
    L = metis.lib()

    def call(dy=(4, 40, 40, 0), pre=(4, 40, 40, 0), dz=(4, 40, 40, 0), act=2, mask=None, db=FAKE, dp=FAKE, zp=FAKE, ws=FAKE, size=1 << 40):
        d, p, z = metis.Mat(dp, *dy), metis.Mat(FAKE, *pre) if pre else None, metis.Mat(zp, *dz) if dz else None
        m = _mask(metis, **mask) if mask is not None else None
        return L.metis_linear_grads(None, C.byref(d), _ref(p), act, _ref(m), _ref(z), db, ws, size)

    assert call(dy=(0, 40, 40, 0), pre=(0, 40, 40, 0), dz=(0, 40, 40, 0), db=None) == 0
    assert call(dp=None) == INVALID and call(pre=None) == INVALID and call(dz=None, db=None) == INVALID and call(act=9) == INVALID and call(zp=None) == INVALID
    assert call(db=FAKE + 2) == INVALID and call(dy=(4, 40, 40, 3)) == INVALID and call(pre=(4, 40, 40, 1)) == INVALID and call(dz=(4, 40, 40, 1)) == INVALID
    for m in BAD_MASKS:
        assert call(mask=m) == INVALID, m
    assert call(dy=(4, 40, 39, 0)) == SHAPE and call(pre=(5, 40, 40, 0)) == SHAPE and call(dz=(4, 41, 41, 0)) == SHAPE and call(pre=(4, 40, 39, 0)) == SHAPE
    assert call(dy=(4, 0, 0, 0), pre=(4, 0, 0, 0), dz=(4, 0, 0, 0)) == SHAPE
    huge = (1 << 28) + 1
    assert call(dy=(4, huge, huge, 0), pre=(4, huge, huge, 0), dz=(4, huge, huge, 0)) == UNSUPPORTED and L.metis_linear_grads_workspace_bytes(4, huge) == 0
    rows = (1000, 40, 40, 0)
    need = L.metis_linear_grads_workspace_bytes(1000, 40)
    assert need > 0 and call(rows, rows, rows, size=need - 1) == WORKSPACE and call(rows, rows, rows, ws=None) == WORKSPACE
    assert call(rows, rows, rows, ws=FAKE + 4) == INVALID and L.metis_linear_grads_workspace_bytes(1, 40) == 0
    assert L.metis_linear_grads(None, None, None, 0, None, None, None, None, 0) == INVALID


def test_layernorm(metis):
    L = metis.lib()

    def call(x=(4, 40, 40, 0), y=(4, 40, 40, 0), w=FAKE, b=FAKE, eps=1e-5, stats=FAKE, xp=FAKE, yp=FAKE):
        a, o = metis.Mat(xp, *x), metis.Mat(yp, *y)
        return L.metis_layernorm(None, C.byref(a), w, b, eps, C.byref(o), stats)

    assert call(x=(0, 40, 40, 0), y=(0, 40, 40, 0)) == 0
    assert call(xp=None) == INVALID and call(yp=None) == INVALID and call(eps=-1e-5) == INVALID and call(eps=NAN) == INVALID
    assert call(w=FAKE + 2) == INVALID and call(b=FAKE + 1) == INVALID and call(stats=FAKE + 4) == INVALID
    assert call(x=(4, 40, 40, 2)) == INVALID and call(y=(4, 40, 40, 1)) == INVALID
    assert call(x=(4, 40, 39, 0)) == SHAPE and call(y=(4, 41, 41, 0)) == SHAPE and call(y=(5, 40, 40, 0)) == SHAPE and call(x=(4, 0, 0, 0), y=(4, 0, 0, 0)) == SHAPE
    huge = (1 << 28) + 1
    assert call(x=(4, huge, huge, 0), y=(4, huge, huge, 0)) == UNSUPPORTED and call(x=(1 << 32, 8, 8, 0), y=(1 << 32, 8, 8, 0)) == UNSUPPORTED
    assert L.metis_layernorm(None, None, None, None, 1e-5, None, None) == INVALID

    def grads(dy=(4, 40, 40, 0), x=(4, 40, 40, 0), dx=(4, 40, 40, 0), add=None, stats=FAKE, w=FAKE, dw=FAKE, db=FAKE, dp=FAKE, xp=FAKE, op=FAKE, ws=FAKE,
              size=1 << 40):
        d, a, o, r = metis.Mat(dp, *dy), metis.Mat(xp, *x), metis.Mat(op, *dx), metis.Mat(FAKE, *add) if add else None
        return L.metis_layernorm_grads(None, C.byref(d), C.byref(a), stats, w, _ref(r), C.byref(o), dw, db, ws, size)

    empty = (0, 40, 40, 0)
    assert grads(empty, empty, empty, dw=None, db=None) == 0
    assert grads(dp=None) == INVALID and grads(xp=None) == INVALID and grads(op=None) == INVALID and grads(stats=None) == INVALID
    assert grads(stats=FAKE + 4) == INVALID and grads(w=FAKE + 2) == INVALID and grads(dw=FAKE + 2) == INVALID and grads(db=FAKE + 2) == INVALID
    assert grads(dy=(4, 40, 40, 1)) == INVALID and grads(dx=(4, 40, 40, 1)) == INVALID and grads(add=(4, 40, 40, 1)) == INVALID and grads(x=(4, 40, 40, 5)) == INVALID
    assert grads(dy=(5, 40, 40, 0)) == SHAPE and grads(dx=(4, 41, 41, 0)) == SHAPE and grads(add=(4, 40, 39, 0)) == SHAPE and grads(x=(4, 40, 39, 0)) == SHAPE
    wide = (4, huge, huge, 0)
    assert grads(wide, wide, wide) == UNSUPPORTED and L.metis_layernorm_grads_workspace_bytes(4, huge) == 0
    assert L.metis_layernorm_grads_workspace_bytes(4, 40) == 0 and L.metis_layernorm_grads_workspace_bytes(512, 16384) == 0
    for shape in ((1281, 40, 40, 0), (700, 16384, 16384, 0), (4, 40000, 40000, 0), (4, 7, 7, 0)):
        need = L.metis_layernorm_grads_workspace_bytes(*shape[:2])
        assert need > 0 and grads(shape, shape, shape, size=need - 1) == WORKSPACE and grads(shape, shape, shape, ws=None) == WORKSPACE
        assert grads(shape, shape, shape, ws=FAKE + 4) == INVALID
    assert L.metis_layernorm_grads(None, None, None, None, None, None, None, None, None, None, 0) == INVALID
