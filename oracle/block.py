"""fp64 oracles of the operators of a block (NumPy, from their definitions): the
norm of a mixer's output with its gate, the residual addition with the norms on
both sides, the gated linear recurrence, and the gated feed-forward
projections, each with its gradients.
"""
import math

import numpy as np


def sigmoid(z):
    return np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))


def inverse_rms(v, eps):
    return 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)


def norm_vjp(v, eps, g):
    """The gradient of v for that of v / rms(v)."""
    r = inverse_rms(v, eps)
    return r * (g - v * r * (g * v * r).mean(-1, keepdims=True))


# ----------------------------------------------------------------------------
def gated_norm(y, z=None, w=None, eps=1e-6, norm_first=False):
    """y, z [B, n, G, d], w [d] or [G, d]."""
    gate = 1.0 if z is None else z * sigmoid(z)
    v = y if norm_first else y * gate
    out = v * inverse_rms(v, eps) * (1.0 if w is None else w)
    return out * gate if norm_first else out


def gated_norm_vjp(y, z, w, eps, norm_first, g):
    """(dy, dz, dw)."""
    ones = np.ones(y.shape[-1]) if w is None else w
    s = np.ones_like(y) if z is None else sigmoid(z)
    gate, slope = (np.ones_like(y), np.zeros_like(y)) if z is None else (z * s, s * (1 + z * (1 - s)))
    v = y if norm_first else y * gate
    hat = v * inverse_rms(v, eps)
    gh = g * gate if norm_first else g
    dv = norm_vjp(v, eps, gh * ones)
    dy = dv if norm_first else dv * gate
    dz = (g * ones * hat if norm_first else dv * y) * slope
    dw = (gh * hat).sum((0, 1) if ones.ndim == 2 else (0, 1, 2))
    return dy, dz, dw


# ----------------------------------------------------------------------------
def residual_norm(x, y, w=None, post=None, scale=None, alpha=1.0, eps=1e-6):
    """(out, r)."""
    u = y if post is None else post * y * inverse_rms(y, eps)
    r = x + alpha * (1.0 if scale is None else scale) * u
    return r * inverse_rms(r, eps) * (1.0 if w is None else w), r


def residual_norm_vjp(x, y, w, post, scale, alpha, eps, g, gr):
    """(dx, dy, dw, dpost, dscale) for the gradients of out and r."""
    one = np.ones(x.shape[-1])
    w1, s1 = one if w is None else w, one if scale is None else scale
    yhat = y * inverse_rms(y, eps)
    u = y if post is None else post * yhat
    r = residual_norm(x, y, w, post, scale, alpha, eps)[1]
    dr = gr + norm_vjp(r, eps, g * w1)
    du = alpha * s1 * dr
    dy = du if post is None else norm_vjp(y, eps, du * post)
    return dr, dy, (g * r * inverse_rms(r, eps)).sum((0, 1)), (du * yhat).sum((0, 1)), (alpha * u * dr).sum((0, 1))


# ----------------------------------------------------------------------------
def glr_gates(x, f, g, decay, fb, gb, c):
    """(r, i, L, a, root): the two gates, log a, a and sqrt(1 - a^2)."""
    r = sigmoid(f + (0.0 if fb is None else fb))
    i = sigmoid(g + (0.0 if gb is None else gb))
    L = -c * np.logaddexp(decay, 0.0) * r
    return r, i, L, np.exp(L), np.sqrt(-np.expm1(2 * L))


def glr(x, f, g, decay, fb=None, gb=None, c=8.0, state=None):
    """x, f, g [B, n, D] -> (every h, the last one), token by token."""
    _, i, _, a, root = glr_gates(x, f, g, decay, fb, gb, c)
    h = np.zeros_like(x[:, 0]) if state is None else state
    hs = np.empty_like(x)
    for t in range(x.shape[1]):
        h = a[:, t] * h + root[:, t] * i[:, t] * x[:, t]
        hs[:, t] = h
    return hs, h


def glr_vjp(x, f, g, decay, fb, gb, c, dy):
    """(dx, df, dg, ddecay, dfb, dgb) from a zero state."""
    r, i, L, a, root = glr_gates(x, f, g, decay, fb, gb, c)
    hs, _ = glr(x, f, g, decay, fb, gb, c)
    before = np.concatenate([np.zeros_like(hs[:, :1]), hs[:, :-1]], 1)
    lam, later = np.empty_like(x), np.zeros_like(x[:, 0])
    for t in reversed(range(x.shape[1])):
        lam[:, t] = dy[:, t] + later
        later = a[:, t] * lam[:, t]
    # root = 0 where L = 0: there L / root and r / root have the limit 0 (r does not vanish otherwise)
    safe = np.where(root > 0, root, 1.0)
    da = lam * a * before
    droot = lam * i * x
    dL = da - np.where(root > 0, droot * a * a / safe, 0.0)
    df, dg = dL * L * (1 - r), lam * root * x * i * (1 - i)
    ddecay = (dL * -c * r).sum((0, 1)) * sigmoid(decay)
    return lam * root * i, df, dg, ddecay, df.sum((0, 1)), dg.sum((0, 1))


# ----------------------------------------------------------------------------
_erfc = np.vectorize(math.erfc, otypes=[float])


def act(p, kind):
    """act(p) and its derivative."""
    if kind == "silu":
        s = sigmoid(p)
        return p * s, s * (1 + p * (1 - s))
    phi = 0.5 * _erfc(-p / math.sqrt(2))      # 1 + erf would lose what is left far below zero
    return p * phi, phi + p * np.exp(-0.5 * p * p) / math.sqrt(2 * math.pi)


def glu(x, wg, wu, kind="silu"):
    """x [B, n, D], wg, wu [F, D] -> [B, n, F]."""
    return act(x @ wg.T, kind)[0] * (x @ wu.T)


def glu_vjp(x, wg, wu, kind, dh):
    """(dx, dwg, dwu, dp, du)."""
    p, u = x @ wg.T, x @ wu.T
    f, d = act(p, kind)
    dp, du = dh * u * d, dh * f
    rows = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    return dp @ wg + du @ wu, rows(dp).T @ rows(x), rows(du).T @ rows(x), dp, du
