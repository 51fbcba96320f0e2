"""Pins of the float64 definition of normalised and turned heads in oracle/memory.py: closed forms and differences."""
import numpy as np

from oracle import memory as om


def test_closed_forms():
    x = np.array([[[[3.0, 4.0, 0.0, 0.0]]]])
    y = om.head_norm(x, None, [[0]], [1.0, 0.5], eps=0.0)
    assert np.allclose(y, [[[[1.2, 1.6, 0, 0]]]])  # root mean square 2.5
    y = om.head_norm(x, [1, 10, 100, 1000], [[1]], [np.pi / 2, np.pi], eps=0.0)
    assert np.allclose(y, [[[[0, -16, 1.2, 0]]]])  # a quarter turn of (0, 2), half a turn of (1, 3)
    # values behind those that are turned stay; zeros are zeros
    y = om.head_norm(x, None, [[7]], [2.0], eps=0.0)
    assert np.allclose(y[..., 2:], 0) and np.allclose(y[..., :2], [[[[1.2 * np.cos(14) - 1.6 * np.sin(14), 1.6 * np.cos(14) + 1.2 * np.sin(14)]]]])
    assert (om.head_norm(np.zeros((1, 1, 1, 4)), None, [[3]], [1.0, 2.0]) == 0).all()


def test_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    q, k = np.repeat(rng.standard_normal((2, 1, 1, 1, 8)), 5, 2)
    f = [1.0, 0.3, 0.1]
    at = np.arange(5)[None]
    d = (om.head_norm(q, None, at + 11, f) * om.head_norm(k, None, at, f)).sum(-1)
    assert np.allclose(d, d[0, 0])


def test_gradients_by_differences():
    rng = np.random.default_rng(1)
    x, w, dy = rng.standard_normal((2, 3, 2, 7)), rng.standard_normal(7), rng.standard_normal((2, 3, 2, 7))
    at, f = rng.integers(0, 100, (2, 3)), [0.5, 0.1]
    dx, dw = om.head_norm_backward(dy, x, w, at, f)
    h = 1e-5
    for got, move in ((dx, lambda d: (x + d, w)), (dw, lambda d: (x, w + d))):
        for i in np.ndindex(got.shape):
            d = np.zeros(got.shape)
            d[i] = h
            up, down = ((om.head_norm(*move(s), at, f) * dy).sum() for s in (d, -d))
            # (third derivatives of order 10: h^2 of them, and rounding 1e-15 / h)
            assert abs((up - down) / (2 * h) - got[i]) < 1e-7
