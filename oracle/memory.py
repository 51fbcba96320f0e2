"""Plain float64 definitions of a policy's memory: layer norm, linear attention with a decay for each head and a gated recurrence,
norms and rotation of heads, forward and backward, one step after the other.  Pinned by closed forms and by differences in tests/test_oracle_memory.py,
tests/test_oracle_recurrence.py and tests/test_oracle_head_norm.py."""
import numpy as np


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """x [N,D] -> (y, mean, rstd)."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * (1.0 if weight is None else weight) + (0.0 if bias is None else bias), mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None):
    """-> (dx, dweight, dbias) for the mean and rstd given."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xh = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    g = dy * (1.0 if weight is None else np.asarray(weight, np.float64))
    D = x.shape[1]
    dx = np.asarray(rstd, np.float64)[:, None] * (g - g.sum(1, keepdims=True) / D - xh * (g * xh).sum(1, keepdims=True) / D)
    return dx, (dy * xh).sum(0), dy.sum(0)


def linear_attention(q, k, v, log_decay, scale, resets=None, state=None):
    """q, k [B,T,H,dk], v [B,T,H,dv], resets [B,T], state [B,H,dk,dv] -> (out [B,T,H,dv], the last state)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, T, H, dk = q.shape
    g = np.exp(np.asarray(log_decay, np.float64))[None, :, None, None]
    S = np.zeros((B, H, dk, v.shape[3])) if state is None else np.array(state, np.float64)
    out = np.zeros((B, T, H, v.shape[3]))
    for t in range(T):
        S = S * g
        if resets is not None:
            S[np.asarray(resets[:, t], bool)] = 0.0
        S = S + k[:, t, :, :, None] * v[:, t, :, None, :]
        out[:, t] = scale * np.einsum("bhd,bhdn->bhn", q[:, t], S)
    return out, S


def linear_attention_backward(dout, q, k, v, log_decay, scale, resets=None, state=None, dstate=None):
    """-> (dq, dk, dv, the gradient of the state before the first step)."""
    dout, q, k, v = (np.asarray(x, np.float64) for x in (dout, q, k, v))
    B, T, H, dk = q.shape
    g = np.exp(np.asarray(log_decay, np.float64))[None, :, None, None]
    S = np.zeros((B, H, dk, v.shape[3])) if state is None else np.array(state, np.float64)
    dq, dk_, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for t in range(T):
        S = S * g
        if resets is not None:
            S[np.asarray(resets[:, t], bool)] = 0.0
        S = S + k[:, t, :, :, None] * v[:, t, :, None, :]
        dq[:, t] = scale * np.einsum("bhdn,bhn->bhd", S, dout[:, t])
    R = np.zeros_like(S) if dstate is None else np.array(dstate, np.float64)
    for t in range(T - 1, -1, -1):
        R = R + scale * q[:, t, :, :, None] * dout[:, t, :, None, :]
        dk_[:, t] = np.einsum("bhdn,bhn->bhd", R, v[:, t])
        dv[:, t] = np.einsum("bhdn,bhd->bhn", R, k[:, t])
        R = R * g
        if resets is not None:
            R[np.asarray(resets[:, t], bool)] = 0.0
    return dq, dk_, dv, R


def _gates(gate):
    """a = 1 / (1 + exp(-gate)) and 1 - a, each to its own last digits."""
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-gate)), 1 / (1 + np.exp(gate))


def gated_recurrence(x, gate, resets=None, state=None, coupled=True):
    """x, gate [B,T,D], resets [B,T], state [B,D] -> (out [B,T,D], the last state)."""
    x, (a, rest) = np.asarray(x, np.float64), _gates(np.asarray(gate, np.float64))
    h = np.zeros((x.shape[0], x.shape[2])) if state is None else np.array(state, np.float64)
    out = np.zeros_like(x)
    for t in range(x.shape[1]):
        h = h * a[:, t]
        if resets is not None:
            h[np.asarray(resets[:, t], bool)] = 0.0
        h = h + (rest[:, t] if coupled else 1.0) * x[:, t]
        out[:, t] = h
    return out, h


def gated_recurrence_backward(dout, x, gate, resets=None, state=None, dstate=None, coupled=True):
    """-> (dx, dgate, the gradient of the state before the first step)."""
    dout, x, (a, rest) = np.asarray(dout, np.float64), np.asarray(x, np.float64), _gates(np.asarray(gate, np.float64))
    out, _ = gated_recurrence(x, gate, resets, state, coupled)
    dx, dgate = np.zeros_like(x), np.zeros_like(x)
    r = np.zeros((x.shape[0], x.shape[2])) if dstate is None else np.array(dstate, np.float64)
    first = np.zeros_like(r) if state is None else np.asarray(state, np.float64)
    for t in range(x.shape[1] - 1, -1, -1):
        cut = np.zeros(x.shape[0], bool) if resets is None else np.asarray(resets[:, t], bool)
        before = np.where(cut[:, None], 0.0, out[:, t - 1] if t else first)
        r = r + dout[:, t]
        dx[:, t] = r * (rest[:, t] if coupled else 1.0)
        dgate[:, t] = r * a[:, t] * rest[:, t] * (before - (x[:, t] if coupled else 0.0))
        r = np.where(cut[:, None], 0.0, r * a[:, t])
    return dx, dgate, r


def _turn(y, positions, frequencies, back=False):
    """The pairs (i, i + r/2) of y [B,T,H,d], r = 2 len(frequencies), turned by positions [B,T] times the frequencies."""
    f = np.asarray(frequencies, np.float64)
    n = len(f)
    angle = (np.asarray(positions, np.float64)[:, :, None] * f)[:, :, None]
    c, s = np.cos(angle), np.sin(-angle if back else angle)
    out = np.array(y, np.float64)
    out[..., :n] = y[..., :n] * c - y[..., n:2 * n] * s
    out[..., n:2 * n] = y[..., n:2 * n] * c + y[..., :n] * s
    return out


def head_norm(x, weight, positions, frequencies, eps=1e-6):
    """x [B,T,H,d], weight [d] or None, positions [B,T], frequencies [r/2] -> y."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, np.float64))
    return _turn(y, positions, frequencies)


def head_norm_backward(dy, x, weight, positions, frequencies, eps=1e-6):
    """-> (dx, dweight)."""
    x = np.asarray(x, np.float64)
    g = _turn(np.asarray(dy, np.float64), positions, frequencies, back=True)
    rstd = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    gw = g * (1.0 if weight is None else np.asarray(weight, np.float64))
    dx = rstd * (gw - x * rstd ** 2 * (gw * x).mean(-1, keepdims=True))
    return dx, (g * x * rstd).sum((0, 1, 2))
