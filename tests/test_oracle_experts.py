"""Pins of the oracle's mixture-of-experts operators: gradients against differences of the forward functions, the E4M3 grid against the library's
type, ties and masks against cases worked by hand."""
import numpy as np
import pytest
import torch

from oracle import experts as oe

CONFIGS = [(s, r) for s in ("softmax", "sigmoid") for r in (False, True)]


@pytest.mark.parametrize("scores,renorm", CONFIGS)
def test_route_grads_are_the_differences(scores, renorm):
    rs = np.random.default_rng(1)
    T, E, k, h = 4, 9, 3, 1e-6
    x = rs.normal(size=(T, E))
    x[1, 4] = -np.inf
    idx, w = oe.route(x, k, scores=scores, renorm=renorm, scale=1.7)
    dw = rs.normal(size=(T, k))
    got = oe.route_grads(x, idx, dw, scores=scores, renorm=renorm, scale=1.7)
    for t in range(T):
        for e in range(E):
            if np.isinf(x[t, e]):
                assert got[t, e] == 0
                continue
            lo, hi = x.copy(), x.copy()
            lo[t, e] -= h
            hi[t, e] += h
            f = [1.7 * oe.chosen_weights(y[t], idx[t], scores, renorm) @ dw[t] for y in (lo, hi)]
            assert abs((f[1] - f[0]) / (2 * h) - got[t, e]) < 1e-8


def test_selection_by_hand():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0, np.nan]])
    assert oe.route(x, 4)[0].tolist() == [[1, 2, 4, 0]]
    assert oe.route(x, 5)[0].tolist() == [[1, 2, 4, 0, -1]]
    assert oe.route(x, 2, bias=np.array([9.0, 0, 0, 99.0, 0, 0]))[0].tolist() == [[0, 1]]
    # groups of two: highest keys 3, 3, 2 (softmax): the first two groups, the tie to the lowest
    assert oe.route(x, 3, groups=3, top_groups=2)[0].tolist() == [[1, 2, 0]]
    assert oe.route(x, 1, groups=3, top_groups=1)[0].tolist() == [[1]]
    # sigmoid: the sum of two; a lone expert counts alone
    assert oe.route(x, 1, groups=3, top_groups=1, scores="sigmoid")[0].tolist() == [[1]]
    assert oe.route(x, 2, valid=np.array([0]))[0].tolist() == [[-1, -1]]
    assert oe.route(np.full((1, 3), -np.inf), 2)[0].tolist() == [[-1, -1]]


def test_plan_by_hand():
    offsets, token, slot = oe.plan(np.array([[2, 0], [-1, 2], [0, 5]]), 4)
    assert offsets.tolist() == [0, 2, 2, 4, 4]
    assert token.tolist() == [0, 2, 0, 1, -1, -1]
    assert slot.tolist() == [[2, 0], [-1, 3], [1, -1]]


def test_e4m3_grid_and_rounding():
    v = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oe.e4m3_values(), v)
    rs = np.random.default_rng(2)
    x = rs.normal(size=(8, 96)) * np.exp(3 * rs.normal(size=(8, 96)))
    x[0, :32] = 0.0
    x[1, :3] = 448.0, 17.0, 18.0                   # no scaling; 17 is half way between 16 and 18
    x[1, 3:32] = 0.0
    x[2, 5] = np.inf
    x[3, 40] = np.nan
    codes, scales = oe.quantize_mx8(x)
    y = oe.dequantize_mx8(codes, scales)
    assert y[1, :3].tolist() == [448.0, 16.0, 18.0] and scales[1, 0] == 127
    assert scales[0, 0] == 0 and not y[0, :32].any()
    assert np.isnan(y[2, :32]).all() and np.isnan(y[3, 32:64]).all() and not np.isnan(y[3, :32]).any()
    fine = ~np.isnan(y)
    scale = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)
    want = torch.from_numpy(np.where(fine, x / scale, 0.0)).to(torch.float32).to(torch.float8_e4m3fn).double().numpy() * scale
    assert np.array_equal(y[fine], want[fine])
    # the block's largest is within 448, and would not be with half the scale
    for r, c in zip(*np.nonzero((scales != 0) & (scales != 255))):
        amax = np.abs(x[r, 32 * c:32 * c + 32]).max()
        s = 2.0 ** (int(scales[r, c]) - 127)
        assert 224 * s < amax <= 448 * s


def test_swiglu_grads_are_the_differences():
    rs = np.random.default_rng(3)
    gu, d, h = 2 * rs.normal(size=(3, 10)), rs.normal(size=(3, 5)), 1e-6
    got = oe.swiglu_grads(gu, d)
    for i in np.ndindex(gu.shape):
        lo, hi = gu.copy(), gu.copy()
        lo[i] -= h
        hi[i] += h
        assert abs(((oe.swiglu(hi) - oe.swiglu(lo)) * d).sum() / (2 * h) - got[i]) < 1e-8


def test_combine_grads_are_the_differences():
    rs = np.random.default_rng(4)
    idx = np.array([[0, 3], [2, -1], [3, 1]])
    offsets, token, slot = oe.plan(idx, 4)
    rows, w, dy, h = rs.normal(size=(6, 7)), rs.normal(size=(3, 2)), rs.normal(size=(3, 7)), 1e-6
    drows, dw = oe.combine_grads(dy, rows, slot, w)
    assert not drows[offsets[-1]:].any() and dw[1, 1] == 0
    for a, g in ((rows, drows), (w, dw)):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            hi = (oe.combine(rows, slot, w) * dy).sum()
            a[i] = keep - h
            lo = (oe.combine(rows, slot, w) * dy).sum()
            a[i] = keep
            assert abs((hi - lo) / (2 * h) - g[i]) < 1e-8
