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
