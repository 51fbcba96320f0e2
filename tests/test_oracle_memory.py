"""Pins of the float64 definitions in oracle/memory.py: closed forms, the sum over pairs of steps, and differences."""
import numpy as np
import pytest

from oracle import memory as om


def test_layer_norm_closed_forms():
    y, mean, rstd = om.layer_norm(np.array([[1.0, -1.0], [5.0, 5.0]]), eps=0.0625)
    assert np.allclose(mean, [0, 5]) and np.allclose(rstd, [1 / np.sqrt(1.0625), 4.0])
    assert np.allclose(y, [[rstd[0], -rstd[0]], [0, 0]])
    x = np.random.default_rng(0).standard_normal((7, 33)) * 3 + 2
    y, _, _ = om.layer_norm(x, eps=0.0)
    assert np.allclose(y.mean(1), 0) and np.allclose((y ** 2).mean(1), 1)
    w, b = np.arange(33.0), -np.arange(33.0)
    assert np.allclose(om.layer_norm(x, w, b, eps=0.0)[0], y * w + b)


def test_layer_norm_gradients_by_differences():
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.standard_normal((4, 9)), rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((4, 9))
    _, mean, rstd = om.layer_norm(x, w, b)
    dx, dw, db = om.layer_norm_backward(dy, x, mean, rstd, w)

    def f(x_, w_, b_):
        return (om.layer_norm(x_, w_, b_)[0] * dy).sum()
    h = 1e-5
    for got, pick in ((dx, lambda d: (x + d, w, b)), (dw, lambda d: (x, w + d, b)), (db, lambda d: (x, w, b + d))):
        for at in np.ndindex(got.shape):
            d = np.zeros(got.shape)
            d[at] = h
            # (third derivatives of order 10: h^2 of them, and rounding 1e-15 / h)
            assert abs((f(*pick(d)) - f(*pick(-d))) / (2 * h) - got[at]) < 1e-7


def _case(rng, B=2, T=9, H=3, dk=4, dv=5):
    q, k, v = rng.standard_normal((B, T, H, dk)), rng.standard_normal((B, T, H, dk)), rng.standard_normal((B, T, H, dv))
    resets = rng.random((B, T)) < 0.25
    return q, k, v, -rng.random(H), resets, rng.standard_normal((B, H, dk, dv))


def test_linear_attention_is_the_sum_over_pairs():
    q, k, v, ld, resets, S0 = _case(np.random.default_rng(2))
    out, last = om.linear_attention(q, k, v, ld, 0.7, resets, S0)
    B, T, H, _ = q.shape
    ep = np.cumsum(resets, 1)
    for b in range(B):
        for h in range(H):
            for t in range(T):
                o = sum(np.exp(ld[h] * (t - j)) * (q[b, t, h] @ k[b, j, h]) * v[b, j, h] for j in range(t + 1) if ep[b, j] == ep[b, t])
                if ep[b, t] == 0:
                    o = o + np.exp(ld[h] * (t + 1)) * (q[b, t, h] @ S0[b, h])
                assert np.allclose(out[b, t, h], 0.7 * o)
            S = sum(np.exp(ld[h] * (T - 1 - j)) * np.outer(k[b, j, h], v[b, j, h]) for j in range(T) if ep[b, j] == ep[b, -1])
            if ep[b, -1] == 0:
                S = S + np.exp(ld[h] * T) * S0[b, h]
            assert np.allclose(last[b, h], S)


def test_linear_attention_without_steps_and_with_one():
    q, k, v, ld, _, S0 = _case(np.random.default_rng(3), T=0)
    out, last = om.linear_attention(q, k, v, ld, 1.0, None, S0)
    assert out.shape[1] == 0 and np.array_equal(last, S0)
    q, k, v, ld, _, S0 = _case(np.random.default_rng(4), T=1)
    out, last = om.linear_attention(q, k, v, ld, 2.0, np.ones((2, 1), bool), S0)
    assert np.allclose(out[:, 0], 2 * (q[:, 0] * k[:, 0]).sum(-1, keepdims=True) * v[:, 0])
    assert np.allclose(last, k[:, 0, :, :, None] * v[:, 0, :, None, :])


@pytest.mark.parametrize("with_state", [True, False])
def test_linear_attention_gradients_by_differences(with_state):
    rng = np.random.default_rng(5)
    q, k, v, ld, resets, S0 = _case(rng)
    dout, dlast = rng.standard_normal(v.shape), rng.standard_normal(S0.shape)
    S0 = S0 if with_state else None
    dq, dk, dv, dS = om.linear_attention_backward(dout, q, k, v, ld, 0.7, resets, S0, dlast)

    def f(q_, k_, v_, s_):
        out, last = om.linear_attention(q_, k_, v_, ld, 0.7, resets, s_)
        return (out * dout).sum() + (last * dlast).sum()
    # f is linear in each of the four: a difference over any distance is the derivative
    for i, got in enumerate((dq, dk, dv, dS)):
        if i == 3 and not with_state:
            continue
        for _ in range(5):
            d = rng.standard_normal(got.shape)
            up, down = [q, k, v, S0], [q, k, v, S0]
            up[i], down[i] = up[i] + d, down[i] - d
            assert abs((f(*up) - f(*down)) / 2 - (got * d).sum()) < 1e-9
