"""Arguments that the mixture-of-experts calls refuse, before anything is enqueued (no GPU needed: the addresses are never read)."""
import ctypes as C
import os

import pytest

FAKE = 1 << 30
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -5


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    m.lib()
    return m


def _router(metis, **kw):
    d = dict(experts=16, k=2, scores=0, groups=1, top_groups=1, renorm=1, scale=1.0)
    d.update(kw)
    return metis.Router(**d)


def test_route(metis):
    L = metis.lib()

    def call(rows=4, cols=16, ld=16, dtype=1, ptr=FAKE, idx=FAKE, w=FAKE, grads=False, **kw):
        m, r = metis.Mat(ptr, rows, cols, ld, dtype), _router(metis, **kw)
        if grads:
            d = metis.Mat(FAKE, rows, cols, ld, 1)
            return L.metis_route_grads(None, C.byref(m), C.byref(r), idx, w, C.byref(d))
        return L.metis_route(None, C.byref(m), C.byref(r), None, None, idx, w)

    for grads in (False, True):
        assert call(rows=0, grads=grads) == 0
        assert call(ptr=None, grads=grads) == INVALID and call(idx=None, grads=grads) == INVALID and call(w=None, grads=grads) == INVALID
        assert call(dtype=7, grads=grads) == INVALID and call(scores=2, grads=grads) == INVALID and call(k=0, grads=grads) == INVALID
        assert call(experts=15, grads=grads) == SHAPE and call(ld=15, grads=grads) == SHAPE
        assert call(experts=513, cols=513, ld=513, grads=grads) == UNSUPPORTED and call(k=17, grads=grads) == UNSUPPORTED
        assert call(rows=1 << 31, grads=grads) == SHAPE
    assert call(groups=3) == INVALID and call(groups=4, top_groups=5) == INVALID and call(groups=4, top_groups=0) == INVALID
    assert call(groups=16, top_groups=1) == INVALID                         # two choices out of one expert
    assert L.metis_route(None, None, None, None, None, None, None) == INVALID
    m, r, d = metis.Mat(FAKE, 4, 16, 16, 1), _router(metis), metis.Mat(FAKE, 4, 8, 16, 1)
    assert L.metis_route_grads(None, C.byref(m), C.byref(r), FAKE, FAKE, C.byref(d)) == SHAPE
    assert L.metis_route_grads(None, C.byref(m), C.byref(r), FAKE, FAKE, None) == INVALID


def test_dispatch(metis):
    L = metis.lib()

    def call(tokens=100, experts=16, k=2, idx=FAKE, offsets=FAKE, token=FAKE, slot=FAKE, ws=FAKE, size=1 << 40):
        p = metis.Plan(offsets, token, slot, tokens, experts, k)
        return L.metis_dispatch(None, idx, C.byref(p), ws, size)

    assert call(idx=None) == INVALID and call(offsets=None) == INVALID and call(token=None) == INVALID and call(slot=None) == INVALID
    assert call(tokens=-1) == INVALID and call(experts=0) == INVALID and call(k=0) == INVALID
    assert call(experts=513) == UNSUPPORTED and call(k=17) == UNSUPPORTED and call(tokens=1 << 31) == SHAPE
    need = L.metis_dispatch_workspace_bytes(100000, 16, 2)
    assert need > 0 and L.metis_dispatch_workspace_bytes(1, 64, 4) == 0
    assert call(tokens=100000, size=need - 1) == WORKSPACE and call(tokens=100000, ws=None) == WORKSPACE
    assert call(tokens=100000, ws=FAKE + 4) == INVALID
    assert L.metis_dispatch(None, FAKE, None, None, 0) == INVALID


def test_checkpoints(metis):
    L = metis.lib()

    def call(rows=4, cols=64, ld=64, dtype=0, ptr=FAKE, codes=FAKE, scales=FAKE, qrows=4, qcols=64, restore=False):
        m, q = metis.Mat(ptr, rows, cols, ld, dtype), metis.Mx8(codes, scales, qrows, qcols)
        return (L.metis_dequantize_mx8(None, C.byref(q), C.byref(m)) if restore else L.metis_quantize_mx8(None, C.byref(m), C.byref(q)))

    for restore in (False, True):
        assert call(ptr=None, restore=restore) == INVALID and call(codes=None, restore=restore) == INVALID
        assert call(scales=None, restore=restore) == INVALID and call(dtype=3, restore=restore) == INVALID
        assert call(qcols=48, restore=restore) == INVALID and call(qrows=5, restore=restore) == SHAPE and call(cols=32, restore=restore) == SHAPE
        assert call(ld=60, restore=restore) == SHAPE and call(ld=68, restore=restore) == SHAPE and call(ptr=FAKE + 8, restore=restore) == SHAPE
        assert call(codes=FAKE + 4, restore=restore) == SHAPE
        assert call(cols=1 << 29, qcols=1 << 29, ld=1 << 29, restore=restore) == UNSUPPORTED
        assert call(rows=0, qrows=0, ptr=None, restore=restore) == 0
    assert L.metis_quantize_mx8(None, None, None) == INVALID and L.metis_dequantize_mx8(None, None, None) == INVALID


def test_swiglu(metis):
    L = metis.lib()

    def call(S=4, F=32, gu=(4, 64, 64, 0), act=(4, 32, 32, 0), q=(4, 64), gp=FAKE, ap=FAKE, grads=False):
        g, a, s = metis.Mat(gp, *gu), metis.Mat(ap, *act), metis.Mx8(FAKE, FAKE, *q)
        if grads:
            return L.metis_swiglu_grads(None, C.byref(s), C.byref(a), C.byref(g), None)
        return L.metis_swiglu(None, C.byref(g), C.byref(a), C.byref(s))

    for grads in (False, True):
        assert call(gp=None, grads=grads) == INVALID and call(ap=None, grads=grads) == INVALID
        assert call(act=(4, 32, 32, 1), grads=grads) == SHAPE and call(act=(4, 48, 48, 0), gu=(4, 96, 96, 0), q=(4, 96), grads=grads) == SHAPE
        assert call(act=(3, 32, 32, 0), grads=grads) == SHAPE and call(act=(4, 32, 36, 0), grads=grads) == SHAPE
        assert call(q=(4, 128), grads=grads) == SHAPE and call(gu=(4, 64, 66, 0), grads=grads) == SHAPE
    assert L.metis_swiglu(None, None, None, None) == INVALID and L.metis_swiglu_grads(None, None, None, None, None) == INVALID


def test_combine(metis):
    L = metis.lib()

    def call(rows=(8, 64, 64, 0), y=(4, 64, 64, 0), tokens=4, k=2, experts=8, rp=FAKE, yp=FAKE, slot=FAKE, w=FAKE, dw=FAKE, drows=None, grads=False):
        r, o, p = metis.Mat(rp, *rows), metis.Mat(yp, *y), metis.Plan(FAKE, FAKE, slot, tokens, experts, k)
        if grads:
            d = metis.Mat(FAKE, *(drows or rows))
            return L.metis_combine_grads(None, C.byref(o), C.byref(r), C.byref(p), w, C.byref(d), dw)
        return L.metis_combine(None, C.byref(r), C.byref(p), w, C.byref(o))

    for grads in (False, True):
        assert call(rp=None, grads=grads) == INVALID and call(yp=None, grads=grads) == INVALID and call(slot=None, grads=grads) == INVALID
        assert call(rows=(8, 64, 64, 2), grads=grads) == INVALID and call(tokens=-1, grads=grads) == INVALID
        assert call(rows=(9, 64, 64, 0), grads=grads) == SHAPE and call(y=(5, 64, 64, 0), grads=grads) == SHAPE
        assert call(y=(4, 32, 64, 0), grads=grads) == SHAPE and call(rows=(8, 64, 63, 0), grads=grads) == SHAPE
        assert call(rows=(68, 64, 64, 0), k=17, grads=grads) == UNSUPPORTED
        assert call(tokens=0, grads=grads) == 0
    assert call(rows=(8, 1 << 29, 1 << 29, 0), y=(4, 1 << 29, 1 << 29, 0)) == UNSUPPORTED
    assert call(w=None, grads=True) == INVALID and call(dw=None, grads=True) == INVALID
    assert call(drows=(8, 64, 64, 1), grads=True) == INVALID and call(drows=(8, 64, 63, 0), grads=True) == SHAPE


def test_products(metis):
    L = metis.lib()

    def product(A=(8, 64, 64, 0), W=(128, 64), C_=(8, 16, 16, 0), tokens=8, k=1, experts=8, gather=0, ap=FAKE, wp=FAKE, ws=FAKE, size=1 << 40, token=FAKE):
        a, w, c = metis.Mat(ap, *A), metis.MxFp4(wp, FAKE, *W), metis.Mat(FAKE, *C_)
        p = metis.Plan(FAKE, token, FAKE, tokens, experts, k)
        return L.metis_experts_product(None, C.byref(a), C.byref(w), C.byref(p), gather, C.byref(c), ws, size)

    assert product(tokens=0) == 0
    assert product(ap=None) == INVALID and product(wp=None) == INVALID and product(tokens=-1) == INVALID and product(A=(8, 64, 64, 5)) == INVALID
    assert product(gather=1, token=None) == INVALID and product(ws=FAKE + 16) == INVALID
    assert product(experts=513) == UNSUPPORTED and product(k=17) == UNSUPPORTED and product(tokens=1 << 31) == SHAPE
    assert product(A=(8, 48, 48, 0), W=(128, 48)) == SHAPE and product(W=(129, 64)) == SHAPE and product(A=(7, 64, 64, 0)) == SHAPE
    assert product(C_=(7, 16, 16, 0)) == SHAPE and product(C_=(8, 16, 15, 0)) == SHAPE and product(A=(8, 64, 60, 0)) == SHAPE
    assert product(A=(8, 64, 68, 0)) == SHAPE and product(wp=FAKE + 8) == SHAPE and product(ap=FAKE + 2) == SHAPE
    need = L.metis_experts_workspace_bytes(8, 8, 8, 16, 64)
    assert need >= 8 * 64 // 2 + 8 * 2 and product(size=need - 1) == WORKSPACE and product(ws=None) == WORKSPACE
    assert L.metis_experts_workspace_bytes(8, 8, 8, 16, 48) == 0

    def wgrad(G=(8, 16, 16, 0), X=(8, 64, 64, 0), dW=(128, 64, 64, 0), tokens=8, k=1, experts=8, gather=0, gp=FAKE, dp=FAKE, ws=FAKE, size=1 << 40):
        g, x, d = metis.Mat(gp, *G), metis.Mat(FAKE, *X), metis.Mat(dp, *dW)
        p = metis.Plan(FAKE, FAKE, FAKE, tokens, experts, k)
        return L.metis_experts_wgrad(None, C.byref(g), C.byref(x), C.byref(p), gather, C.byref(d), ws, size)

    assert wgrad(gp=None) == INVALID and wgrad(dp=None) == INVALID and wgrad(ws=FAKE + 16) == INVALID
    assert wgrad(G=(8, 12, 16, 0), dW=(96, 64, 64, 0)) == SHAPE and wgrad(G=(7, 16, 16, 0)) == SHAPE and wgrad(X=(4, 64, 64, 0)) == SHAPE
    assert wgrad(dW=(127, 64, 64, 0)) == SHAPE and wgrad(dW=(128, 64, 63, 0)) == SHAPE and wgrad(G=(8, 16, 20, 0)) == SHAPE
    huge = 1 << 29
    assert wgrad(X=(8, huge, huge, 0), dW=(128, huge, huge, 0)) == UNSUPPORTED and L.metis_experts_wgrad_workspace_bytes(8, 8, 16, huge) == 0
    assert product(A=(8, huge, huge, 0), W=(128, huge)) == UNSUPPORTED and L.metis_experts_workspace_bytes(8, 8, 8, 16, huge) == 0
    need = L.metis_experts_wgrad_workspace_bytes(8, 8, 16, 64)
    assert need > 0 and wgrad(size=need - 1) == WORKSPACE and wgrad(ws=None) == WORKSPACE

    def quantize_t(A=(64, 16, 16, 0), out=(32, 32), groups=2, ap=FAKE, codes=FAKE):
        a, o = metis.Mat(ap, *A), metis.MxFp4(codes, FAKE, *out)
        return L.metis_quantize_mx_t(None, C.byref(a), groups, C.byref(o))

    assert quantize_t(ap=None) == INVALID and quantize_t(codes=None) == INVALID and quantize_t(groups=0) == INVALID
    assert quantize_t(groups=3) == SHAPE and quantize_t(groups=4) == SHAPE and quantize_t(out=(16, 32)) == SHAPE
    assert quantize_t(A=(64, 12, 16, 0), out=(24, 32)) == SHAPE and quantize_t(codes=FAKE + 8) == SHAPE and quantize_t(A=(64, 16, 20, 0)) == SHAPE
    assert L.metis_quantize_mx_t(None, None, 1, None) == INVALID and L.metis_experts_product(None, None, None, None, 0, None, None, 0) == INVALID
