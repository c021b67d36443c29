"""GPU parity of the layer norm and its gradients with the fp64 oracle.

u = 2^-24.  A row's sums have at most 64 roundings on any element's way (up to 40 elements of a thread one after the other, then the wave's and the
workgroup's lanes): the mean is off by 64 u mean|x|, the variance by 64 u and three roundings of each term, rstd by half of that and four roundings.  The
columns' sums have at most T + 160.  Results round once more: 2^-8 for bf16, u for fp32."""
import numpy as np
import pytest
import torch

from oracle import epilogue as oep

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: u}


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def _f64(t):
    return t.double().cpu().numpy()


def _inputs(T, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, D), generator=g) * torch.exp(torch.randn((T, 1), generator=g)) + 3 * torch.randn((T, 1), generator=g)
    x[:, ::101] *= 10
    dy, add = torch.randn((T, D), generator=g), torch.randn((T, D), generator=g)
    w, b = 1 + 0.3 * torch.randn(D, generator=g), 0.3 * torch.randn(D, generator=g)
    return x.to(dtype), dy.to(dtype), add.to(dtype), w, b


def _offset(t, pad):
    whole = torch.full((t.shape[0], t.shape[1] + 2 * pad), 7.0, dtype=t.dtype, device="cuda")
    inner = whole[:, pad:pad + t.shape[1]]
    inner.copy_(t)
    return whole, inner


SIZES = [(1, 1), (2, 2), (1, 7), (5, 8), (9, 130), (70, 512), (33, 513), (3, 1000), (17, 2048), (40, 2057), (64, 4096), (5, 4100), (3, 8192), (4, 8200),
         (2, 16384), (3, 16390), (2, 40000), (1200, 24), (1500, 600)]


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layernorm(metis, T, D, dtype):
    x, _, _, w, b = _inputs(T, D, dtype, T + D)
    x64 = _f64(x)
    for weight, bias, eps, pad, inplace in ((w, b, 1e-5, 0, False), (w, b, 1e-3, 3, True), (None, None, 1e-5, 0, False), (w, None, 1e-5, 1, False)):
        whole, xd = _offset(x, pad)
        wy, y = (whole, xd) if inplace else _offset(x * 0, pad)
        stats = torch.empty((T, 2), device="cuda")
        up = lambda v: v.cuda() if v is not None else None
        assert metis.layernorm(xd, y, up(weight), up(bias), eps, stats) is y
        ref, rstats = oep.layernorm(x64, None if weight is None else _f64(weight), None if bias is None else _f64(bias), np.float32(eps).astype(np.float64))
        mean, rstd = rstats[:, :1], rstats[:, 1:]
        em = 64 * u * np.abs(x64).mean(1, keepdims=True) + u * np.abs(mean)
        # a mean off by em adds em^2 to the variance
        er = 0.5 * (70 * u + em * em * rstd * rstd) + 4 * u
        ww = np.ones(D) if weight is None else np.abs(_f64(weight))
        xh = (x64 - mean) * rstd
        err = ww * (np.abs(xh) * (er + 4 * u) + rstd * em * (1 + er)) + 2 * u * np.abs(ref)
        if bias is not None:
            err = err + u * np.abs(_f64(bias))
        got = _f64(y)
        assert np.all(np.abs(got - ref) <= err + ROUND[dtype] * (np.abs(ref) + err)), float(np.max(np.abs(got - ref) - err))
        s = _f64(stats)
        assert np.all(np.abs(s[:, :1] - mean) <= em) and np.all(np.abs(s[:, 1:] - rstd) <= er * rstd)
        if pad:
            assert (wy[:, :pad] == 7).all() and (wy[:, D + pad:] == 7).all()
        if not inplace:
            again = metis.layernorm(xd, torch.empty_like(y), up(weight), up(bias), eps)
            assert torch.equal(again, y)                       # without statistics, the same bits


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layernorm_grads(metis, T, D, dtype):
    x, dy, add, w, _ = _inputs(T, D, dtype, T + 2 * D)
    stats = torch.from_numpy(oep.layernorm(_f64(x), None, None, 1e-5)[1]).float()
    x64, dy64, st = _f64(x), _f64(dy), _f64(stats)
    for weight, plus, pad, inplace, columns in ((w, None, 0, None, True), (w, add, 3, "dy", True), (None, add, 0, "add", True), (w, add, 1, "x", False)):
        (wd, d), (wx, xd), (wa, ad) = _offset(dy, pad), _offset(x, pad), _offset(add, pad)
        wo, dx = {"dy": (wd, d), "x": (wx, xd), "add": (wa, ad), None: _offset(x * 0, pad)}[inplace]
        dw, db = (torch.full((D,), 3.0, device="cuda") for _ in range(2))
        wgt = weight.cuda() if weight is not None else None
        keep = d.clone(), xd.clone(), ad.clone()
        assert metis.layernorm_grads(d, xd, stats.cuda(), dx, wgt, dw if columns else None, db if columns else None, ad if plus is not None else None) is dx
        rdx, rdw, rdb = oep.layernorm_grads(dy64, x64, st, None if weight is None else _f64(weight), None if plus is None else _f64(add))
        mean, rstd = st[:, :1], st[:, 1:]
        xh, g = (x64 - mean) * rstd, dy64 * (1.0 if weight is None else _f64(weight))
        mg, mgx = np.abs(g).mean(1, keepdims=True), np.abs(g * xh).mean(1, keepdims=True)
        err = rstd * (8 * u * (np.abs(g) + mg + np.abs(xh) * mgx) + 66 * u * mg + np.abs(xh) * 70 * u * mgx) + 2 * u * np.abs(rdx)
        if plus is not None:
            err = err + u * np.abs(_f64(add))
        got = _f64(dx)
        assert np.all(np.abs(got - rdx) <= err + ROUND[dtype] * (np.abs(rdx) + err))
        if columns:
            assert np.all(np.abs(_f64(dw) - rdw) <= (T + 164) * u * np.abs(dy64 * xh).sum(0) + 1e-37)
            assert np.all(np.abs(_f64(db) - rdb) <= (T + 160) * u * np.abs(dy64).sum(0) + 1e-37)
            again = [torch.empty_like(dw) for _ in range(2)]
            out = torch.empty_like(x, device="cuda")
            metis.layernorm_grads(keep[0], keep[1], stats.cuda(), out, wgt, again[0], again[1], keep[2] if plus is not None else None)
            assert torch.equal(again[0], dw) and torch.equal(again[1], db) and torch.equal(out, dx)      # the same bits every time
            metis.layernorm_grads(keep[0], keep[1], stats.cuda(), out, wgt, None, again[1])              # one of the two alone
            assert torch.equal(again[1], db)
        if pad:
            assert (wo[:, :pad] == 7).all() and (wo[:, D + pad:] == 7).all()


@pytest.mark.parametrize("T,D", [(255, 65), (256, 64), (256, 4090), (512, 10), (512, 9000), (513, 9000), (1280, 63), (1281, 63), (129, 9), (256, 7), (31, 16390)])
def test_layernorm_grads_near_the_rules(metis, T, D):
    """The same sums and the same rows wherever dx goes: the columns' sums read dy and x before dx takes the place of either."""
    x, dy, add, w, _ = _inputs(T, D, torch.float32, T * D)
    stats = torch.from_numpy(oep.layernorm(_f64(x), None, None, 1e-5)[1]).float()
    xd, d, a, wgt = (t.cuda() for t in (x, dy, add, w))
    first = None
    for place in (None, "dy", "x", "add", "add and x"):
        xs, ds, as_ = xd.clone(), d.clone(), a.clone()
        if place == "add and x":
            as_ = xs
        dx = {None: torch.empty_like(xd), "dy": ds, "x": xs, "add": as_, "add and x": xs}[place]
        dw, db = torch.empty_like(wgt), torch.empty_like(wgt)
        metis.layernorm_grads(ds, xs, stats.cuda(), dx, wgt, dw, db, as_)
        first = first or (dx, dw, db)
        assert torch.equal(dw, first[1]) and torch.equal(db, first[2]) and (place == "add and x" or torch.equal(dx, first[0]))
    xh, dy64 = (_f64(x) - _f64(stats)[:, :1]) * _f64(stats)[:, 1:], _f64(dy)
    assert np.all(np.abs(_f64(first[1]) - (dy64 * xh).sum(0)) <= (T + 164) * u * np.abs(dy64 * xh).sum(0) + 1e-37)
    assert np.all(np.abs(_f64(first[2]) - dy64.sum(0)) <= (T + 160) * u * np.abs(dy64).sum(0) + 1e-37)


@pytest.mark.parametrize("T,D", [(5, 2057), (1300, 77), (3, 9), (2, 5), (40, 9003)])
def test_missing_values_stay_in_their_columns(metis, T, D):
    for at in {max(D - 9, 0), D // 8 * 8 - 1 if D > 8 else 0, D - 1}:
        x, dy, stats = torch.zeros((T, D), device="cuda"), torch.ones((T, D), device="cuda"), torch.tensor([[-1.0, 1.0]], device="cuda").repeat(T, 1)
        x[1, at] = float("nan")
        dw, db, dx = torch.empty(D, device="cuda"), torch.empty(D, device="cuda"), torch.empty_like(x)
        metis.layernorm_grads(dy, x, stats, dx, None, dw, db)
        assert torch.isnan(dw).sum() == 1 and torch.isnan(dw[at]) and (dw[torch.arange(D, device="cuda") != at] == T).all() and (db == T).all()
        rows = torch.isnan(dx).any(1)
        assert rows.sum() == 1 and rows[1]


def test_gradients_are_the_forward_pass_differences(metis):
    """fp32; a step h: results rounded to 2^-23 of magnitudes up to 5, their 30 products with dy summed, over 2 h; and h^2 / 6 of third derivatives of
    rows of unit scale."""
    T, D, h = 3, 30, 2.0 ** -8
    g = torch.Generator().manual_seed(4)
    x, dy, w, b = (torch.randn(s, generator=g) for s in ((T, D), (T, D), (D,), (D,)))
    cuda = lambda *t: [v.cuda() for v in t]

    def f(x_, w_, b_):
        xd, wd, bd = cuda(x_, w_, b_)
        return (metis.layernorm(xd, torch.empty_like(xd), wd, bd).double().cpu() * dy.double()).sum().item()

    xd, dyd, wd, bd = cuda(x, dy, w, b)
    stats, dx, dw, db = torch.empty((T, 2), device="cuda"), torch.empty_like(xd), torch.empty_like(wd), torch.empty_like(bd)
    metis.layernorm(xd, torch.empty_like(xd), wd, bd, stats=stats)
    metis.layernorm_grads(dyd, xd, stats, dx, wd, dw, db)
    for arg, grad in ((0, dx), (1, dw), (2, db)):
        for at in list(np.ndindex(*grad.shape))[::3]:
            lo, hi = [v.clone() for v in (x, w, b)], [v.clone() for v in (x, w, b)]
            lo[arg][at] -= h
            hi[arg][at] += h
            assert abs((f(*hi) - f(*lo)) / (2 * h) - grad[at].item()) < 3e-3


def test_rows_without_spread_and_missing_values(metis):
    x = torch.full((4, 300), 2.5, device="cuda")
    x[1] = 0.0
    x[2, 7] = float("nan")
    x[3] = torch.randn(300)
    stats = torch.empty((4, 2), device="cuda")
    y = metis.layernorm(x, torch.empty_like(x), None, None, 1e-5, stats).cpu()
    assert (y[:2] == 0).all() and torch.isnan(y[2]).all() and torch.isfinite(y[3]).all()        # a row keeps its NaN to itself
    assert abs(stats[0, 1].item() - 1e-5 ** -0.5) < 1e-3
    dx = metis.layernorm_grads(torch.ones_like(x), x, stats, torch.empty_like(x)).cpu()
    assert torch.isfinite(dx[:2]).all() and torch.isnan(dx[2]).all() and torch.isfinite(dx[3]).all()


def test_rows_far_from_zero(metis):
    """A mean a thousand times the spread: the variance comes from differences, so rstd keeps its accuracy (bound of test_layernorm)."""
    x = 1000 + torch.randn((8, 4096), generator=torch.Generator().manual_seed(1))
    stats = torch.empty((8, 2), device="cuda")
    metis.layernorm(x.cuda(), torch.empty((8, 4096), device="cuda"), stats=stats)
    _, ref = oep.layernorm(_f64(x), None, None, 1e-5)
    em = 64 * u * 1000
    assert np.all(np.abs(_f64(stats)[:, 1] / ref[:, 1] - 1) <= 0.5 * (70 * u + (em * ref[:, 1]) ** 2) + 4 * u)


def test_no_rows(metis):
    e, s = torch.empty((0, 40), device="cuda"), torch.empty((0, 2), device="cuda")
    metis.layernorm(e, e, stats=s)
    dw, db = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    metis.layernorm_grads(e, e, s, e, dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
