"""Plain float64 definitions of a policy's memory: layer norm and linear attention with a decay for each head, forward and
backward, one step after the other.  Pinned by closed forms and by differences in tests/test_oracle_memory.py."""
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
