"""The oracle of the operators around the products: derivatives against differences, and masks against what they have to be."""
import numpy as np
import pytest

from oracle import epilogue as oep

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("name", ACTS)
def test_slopes_are_the_activations_differences(name):
    z = np.random.default_rng(1).standard_normal(2000) * 3
    z = z[np.abs(z) > 1e-3]                                     # (relu's corner)
    h = 1e-5
    diff = (oep.act(name, z + h) - oep.act(name, z - h)) / (2 * h)
    assert np.max(np.abs(sum(oep.slope_terms(name, z)) - diff)) < 1e-8


def test_activations_at_known_points():
    z = np.array([-1.0, 0.0, 1.0])
    assert np.allclose(oep.act("gelu", z), [-0.15865525393145707, 0.0, 0.8413447460685429], atol=1e-15)
    assert np.allclose(oep.act("silu", z), [-0.2689414213699951, 0.0, 0.7310585786300049], atol=1e-15)
    assert np.allclose(oep.act("gelu_tanh", z), 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))), atol=1e-15)


def test_layernorm_gradients_are_the_differences():
    r = np.random.default_rng(2)
    x, w, b, dy = r.standard_normal((5, 17)) + 2, r.standard_normal(17), r.standard_normal(17), r.standard_normal((5, 17))
    f = lambda x_, w_, b_: float((oep.layernorm(x_, w_, b_, 1e-5)[0] * dy).sum())
    dx, dw, db = oep.layernorm_grads(dy, x, oep.layernorm(x, w, b, 1e-5)[1], w, None)
    h = 1e-6
    for arg, grad in ((0, dx), (1, dw), (2, db)):
        for at in np.ndindex(*grad.shape):
            lo, hi = [v.copy() for v in (x, w, b)], [v.copy() for v in (x, w, b)]
            lo[arg][at] -= h
            hi[arg][at] += h
            assert abs((f(*hi) - f(*lo)) / (2 * h) - grad[at]) < 1e-7


def test_masks():
    rows, cols = 4000, 203
    for p in (0.1, 0.5, 0.9):
        m = oep.mask(p, 77, 3, np.arange(rows), cols)
        t = int(np.floor(65536 * p + 0.5))
        kept = (m > 0).mean()
        assert abs(kept - (1 - t / 65536)) < 5 * np.sqrt(p * (1 - p) / (rows * cols))
        assert set(np.unique(m)) == {0.0, 65536 / (65536 - t)}
        # every one of a block's eight numbers, and every row and column, drops its share (5.5 deviations of some 200 and 4000 counts)
        for axis, n in ((0, rows), (1, cols)):
            assert np.max(np.abs((m > 0).mean(axis) - (1 - t / 65536))) < 5.5 * np.sqrt(p * (1 - p) / n)
    a = oep.mask(0.5, 77, 3, np.arange(64), cols)
    assert np.array_equal(oep.mask(0.5, 77, 3 + (1 << 32), np.arange(64), cols), a)             # the step counts modulo 2^32
    for other in (oep.mask(0.5, 78, 3, np.arange(64), cols), oep.mask(0.5, 77, 4, np.arange(64), cols), oep.mask(0.5, 77 + (1 << 32), 3, np.arange(64), cols)):
        assert abs((a != other).mean() - 0.5) < 0.03
    assert np.array_equal(oep.mask(0.5, 77, 3, np.arange(64), 50), a[:, :50])                   # the width changes nothing
    assert (oep.mask(0.0, 1, 0, np.arange(9), 9) == 1).all()
