"""Pins of the float64 definition of a gated recurrence in oracle/memory.py: closed forms, the sum over pairs of steps, and differences."""
import numpy as np
import pytest

from oracle import memory as om


def test_closed_forms():
    # a gate of 0 keeps a half; one that is wide open keeps everything, one that is shut nothing
    x = np.ones((1, 4, 3))
    gate = np.broadcast_to([0.0, 800.0, -800.0], (1, 4, 3))
    out, last = om.gated_recurrence(x, gate, state=np.full((1, 3), 3.0))
    assert np.allclose(out[0, :, 0], 1 + 2 * 0.5 ** np.arange(1, 5)) and np.allclose(out[0, :, 1], 3) and np.allclose(out[0, :, 2], 1)
    assert np.array_equal(out[:, -1], last)
    out, _ = om.gated_recurrence(x, gate, coupled=False)
    assert np.allclose(out[0, :, 0], 2 - 0.5 ** np.arange(4)) and np.allclose(out[0, :, 1], np.arange(1, 5)) and np.allclose(out[0, :, 2], 1)
    out, last = om.gated_recurrence(x, gate, resets=np.array([[0, 0, 1, 0]], bool), state=np.full((1, 3), np.inf))
    assert np.allclose(out[0, 2:, 1], 0) and np.allclose(out[0, 2:, 0], [0.5, 0.75]) and np.isfinite(last).all()
    out, last = om.gated_recurrence(x[:, :0], gate[:, :0], state=np.full((1, 3), 3.0))
    assert out.shape == (1, 0, 3) and np.all(last == 3)


@pytest.mark.parametrize("coupled", [True, False])
def test_is_the_sum_over_pairs_of_steps(coupled):
    rng = np.random.default_rng(0)
    x, gate, state = rng.standard_normal((2, 9, 4)), rng.standard_normal((2, 9, 4)) * 2, rng.standard_normal((2, 4))
    resets = rng.random((2, 9)) < 0.25
    out, _ = om.gated_recurrence(x, gate, resets, state, coupled)
    a = 1 / (1 + np.exp(-gate))
    ep = np.cumsum(resets, 1)
    for b in range(2):
        for t in range(9):
            h = sum(np.prod(a[b, j + 1:t + 1], 0) * ((1 - a[b, j]) if coupled else 1) * x[b, j] for j in range(t + 1) if ep[b, j] == ep[b, t])
            if ep[b, t] == 0:
                h = h + np.prod(a[b, :t + 1], 0) * state[b]
            assert np.allclose(out[b, t], h)


@pytest.mark.parametrize("coupled", [True, False])
@pytest.mark.parametrize("with_state", [True, False])
def test_gradients_by_differences(coupled, with_state):
    rng = np.random.default_rng(1)
    x, gate, state = rng.standard_normal((2, 9, 4)), rng.standard_normal((2, 9, 4)) * 2, rng.standard_normal((2, 4)) if with_state else None
    resets = rng.random((2, 9)) < 0.2
    dout, dlast = rng.standard_normal(x.shape), rng.standard_normal((2, 4))
    dx, dgate, dstate = om.gated_recurrence_backward(dout, x, gate, resets, state, dlast, coupled)

    def f(x_, gate_, state_):
        out, last = om.gated_recurrence(x_, gate_, resets, state_, coupled)
        return (out * dout).sum() + (last * dlast).sum()
    h = 1e-5
    for i, got in enumerate((dx, dgate, dstate)):
        if i == 2 and not with_state:
            continue
        for at in np.ndindex(got.shape):
            up, down = [x, gate, state], [x, gate, state]
            d = np.zeros(got.shape)
            d[at] = h
            up[i], down[i] = up[i] + d, down[i] - d
            # (third derivatives of order 10: h^2 of them, and rounding 1e-15 / h)
            assert abs((f(*up) - f(*down)) / (2 * h) - got[at]) < 1e-7
