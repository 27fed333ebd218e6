"""fp64 oracles of the operators around the attention (NumPy, from their
definitions): the short causal convolution, the norm and rotation of queries
and keys, and the selective state space scan, each with its gradients.  The
scan is the plain token by token recurrence and its adjoint.
"""
import numpy as np


def sigmoid(z):
    return 1.0 / (1.0 + np.exp(-z))


def conv(x, w, bias=None, silu=True, state=None):
    """x [B, n, D], w [D, K] -> (y, z, the last K-1 inputs)."""
    B, n, D = x.shape
    K = w.shape[1]
    past = np.concatenate([np.zeros((B, K - 1, D)) if state is None else state, x], 1)
    z = np.zeros((B, n, D))
    for t in range(n):
        for j in range(K):
            z[:, t] += w[:, j] * past[:, t + j]
    if bias is not None:
        z = z + bias
    return (z * sigmoid(z) if silu else z), z, past[:, n:]


def conv_vjp(x, w, bias, silu, dy):
    """Gradients (dx, dw, dbias) for dy [B, n, D]."""
    B, n, D = x.shape
    K = w.shape[1]
    z = conv(x, w, bias, False)[0]
    s = sigmoid(z)
    dz = dy * (s * (1 + z * (1 - s)) if silu else 1.0)
    dx, dw = np.zeros_like(x), np.zeros_like(w)
    for t in range(n):
        for j in range(K):
            i = t - K + 1 + j
            if i >= 0:
                dx[:, i] += w[:, j] * dz[:, t]
                dw[:, j] += (dz[:, t] * x[:, i]).sum(0)
    return dx, dw, dz.sum((0, 1))


def pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(u, cos, sin, interleaved):
    """u [..., d], cos and sin broadcastable to [..., rot/2]."""
    a, b = pairs(2 * cos.shape[-1], interleaved)
    y = u.copy()
    y[..., a] = u[..., a] * cos - u[..., b] * sin
    y[..., b] = u[..., b] * cos + u[..., a] * sin
    return y


def norm_rope(x, w, cos, sin, eps, interleaved=False):
    """x [B, n, H, d], cos and sin [B, n, rot/2] -> [B, H, n, d]."""
    x = x.transpose(0, 2, 1, 3)
    u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(u * (1.0 if w is None else w), cos[:, None], sin[:, None], interleaved)


def norm_rope_vjp(x, w, cos, sin, eps, interleaved, dy):
    """Gradients (dx [B, n, H, d], dw [d]) for dy [B, H, n, d]."""
    x = x.transpose(0, 2, 1, 3)
    w = np.ones(x.shape[-1]) if w is None else w
    inv = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    g = rotate(dy, cos[:, None], -sin[:, None], interleaved)
    xhat = x * inv
    gw = g * w
    dx = inv * (gw - xhat * (gw * xhat).mean(-1, keepdims=True))
    return dx.transpose(0, 2, 1, 3), (g * xhat).sum((0, 1, 2))


def softplus(x):
    return np.logaddexp(x, 0.0)


def ssm(x, dt, A, Bm, Cm, D=None, dt_bias=None, use_softplus=True, state=None):
    """x [B, n, H, P], dt [B, n, H], Bm, Cm [B, n, G, N] -> (y, the state [B, H, N, P])."""
    B, n, H, P = x.shape
    G, N = Bm.shape[2:]
    Bm, Cm = (np.repeat(m, H // G, 2) for m in (Bm, Cm))
    raw = dt if dt_bias is None else dt + dt_bias
    dt = softplus(raw) if use_softplus else raw
    h = np.zeros((B, H, N, P)) if state is None else state.astype(np.float64).copy()
    y = np.zeros_like(x)
    for t in range(n):
        h = np.exp(dt[:, t] * A)[..., None, None] * h + (
            dt[:, t, :, None, None] * Bm[:, t, :, :, None] * x[:, t, :, None, :])
        y[:, t] = (Cm[:, t, :, :, None] * h).sum(2)
    return y + (0.0 if D is None else D[:, None] * x), h


def ssm_vjp(x, dt, A, Bm, Cm, D, dt_bias, use_softplus, dy, absolute=False):
    """Gradients (dx, ddt, dA, dBm, dCm, dD, ddt_bias) for dy, from a zero state.
    absolute: the same sums over the absolute values of their terms, the scale
    of their rounding errors."""
    if absolute:
        x, Bm, Cm, dy = (np.abs(m) for m in (x, Bm, Cm, dy))
        D = None if D is None else np.abs(D)
    B, n, H, P = x.shape
    G, N = Bm.shape[2:]
    kb, kc = (np.repeat(m, H // G, 2) for m in (Bm, Cm))
    raw = dt if dt_bias is None else dt + dt_bias
    step = softplus(raw) if use_softplus else raw
    decay = np.exp(step * A)
    states = [np.zeros((B, H, N, P))]
    for t in range(n):
        states.append(decay[:, t, :, None, None] * states[-1] +
                      step[:, t, :, None, None] * kb[:, t, :, :, None] * x[:, t, :, None, :])
    g = np.zeros((B, H, N, P))
    dx, dstep = np.zeros_like(x), np.zeros_like(step)
    db, dc = np.zeros_like(kb), np.zeros_like(kc)
    da = np.zeros_like(step)
    for t in reversed(range(n)):
        g = g + kc[:, t, :, :, None] * dy[:, t, :, None, :]
        dc[:, t] = (states[t + 1] * dy[:, t, :, None, :]).sum(-1)
        db[:, t] = step[:, t, :, None] * (g * x[:, t, :, None, :]).sum(-1)
        du = (g * kb[:, t, :, :, None]).sum(2)
        dx[:, t] = step[:, t, :, None] * du + (0.0 if D is None else D[:, None] * dy[:, t])
        g = decay[:, t, :, None, None] * g
        da[:, t] = (g * states[t]).sum((-1, -2))
        dstep[:, t] = (np.abs(A) if absolute else A) * da[:, t] + (du * x[:, t]).sum(-1)
    ddt = dstep * (sigmoid(raw) if use_softplus else 1.0)
    dA = (np.abs(step) * da if absolute else step * da).sum((0, 1))
    db, dc = (m.reshape(B, n, G, H // G, N).sum(3) for m in (db, dc))
    return dx, ddt, dA, db, dc, (dy * x).sum((0, 1, 3)), ddt.sum((0, 1))
