"""Pins of the fp64 oracles of the operators around the attention: worked
examples, closed forms, and every gradient against central differences.

Differences: the functions are smooth and of order one, so with a step of 1e-5
the truncation is about 1e-10 and the rounding 1e-11 of a sum of order ten:
1e-7 of the gradient's scale is a wide bar that any wrong term exceeds.  CPU only.
"""
import numpy as np
import pytest

from oracle import mixer as O

STEP, BAR = 1e-5, 1e-7


def _rng(seed):
    return np.random.default_rng(seed)


def _by_differences(f, args, i, dy):
    """d sum(dy f(args)) / d args[i], element by element."""
    x = args[i]
    out = np.zeros_like(x)
    for at in np.ndindex(*x.shape):
        def val(e):
            y = x.copy()
            y[at] += e
            return (dy * f(*args[:i], y, *args[i + 1:])).sum()
        out[at] = (val(STEP) - val(-STEP)) / (2 * STEP)
    return out


def _close(got, ref):
    assert got.shape == ref.shape
    assert np.abs(got - ref).max() <= BAR * max(1.0, np.abs(ref).max())


def test_conv_by_hand():
    x = np.array([[[1.0], [2.0], [3.0]]])
    w = np.array([[10.0, 1.0]])
    y, _, last = O.conv(x, w, np.array([0.5]), False)
    assert y[0, :, 0].tolist() == [1.5, 12.5, 23.5] and last[0, :, 0].tolist() == [3.0]
    y, _, last = O.conv(x[:, :1], np.array([[100.0, 10.0, 1.0]]), None, False, np.array([[[7.0], [8.0]]]))
    assert y[0, 0, 0] == 781.0 and last[0, :, 0].tolist() == [8.0, 1.0]


def test_rotation_by_hand():
    x = np.array([3.0, 0.0, 4.0, 0.0]).reshape(1, 1, 1, 4)
    quarter, none = np.array([[[0.0, 1.0]]]), np.array([[[1.0, 0.0]]])
    y = O.norm_rope(x, None, quarter, none, 0.0)            # pair (0, 2) by a quarter turn, norm 5 / sqrt 4
    assert np.allclose(y.ravel(), np.array([-4.0, 0.0, 3.0, 0.0]) / 2.5)
    y = O.norm_rope(x, np.full(4, 0.5), quarter, none, 0.0, True)   # pair (0, 1); unit length
    assert np.allclose(y.ravel(), np.array([0.0, 3.0, 4.0, 0.0]) / 5)


def test_scan_closed_forms():
    n = 7
    one = np.ones((1, n, 1, 1))
    zero = np.zeros((1, n, 1))
    # A = 0: running sums; dt = ln 2 with the softplus of 0
    y, h = O.ssm(one, zero, np.zeros(1), one, one)
    assert np.allclose(y.ravel(), np.log(2) * np.arange(1, n + 1)) and np.isclose(h.item(), n * np.log(2))
    # a geometric sum: dt = 1, decay e^-1, plus the skip
    y, _ = O.ssm(one, zero + 1, np.array([-1.0]), one, one, np.array([3.0]), None, False)
    assert np.allclose(y.ravel(), 3 + np.cumsum(np.exp(-np.arange(n))))
    # a state carried over a cut
    r = _rng(0)
    x, dt, A = r.standard_normal((2, 9, 4, 3)), r.standard_normal((2, 9, 4)), -r.random(4)
    Bm, Cm = r.standard_normal((2, 2, 9, 2, 5))
    y, h = O.ssm(x, dt, A, Bm, Cm)
    y1, h1 = O.ssm(x[:, :4], dt[:, :4], A, Bm[:, :4], Cm[:, :4])
    y2, h2 = O.ssm(x[:, 4:], dt[:, 4:], A, Bm[:, 4:], Cm[:, 4:], state=h1)
    assert np.allclose(np.concatenate([y1, y2], 1), y) and np.allclose(h2, h)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("K", [2, 3, 4])
def test_conv_gradients(K, silu):
    r = _rng(K)
    x, w, b, dy = r.standard_normal((2, 5, 3)), r.standard_normal((3, K)), r.standard_normal(3), r.standard_normal((2, 5, 3))
    grads = O.conv_vjp(x, w, b, silu, dy)
    for i in range(3):
        _close(grads[i], _by_differences(lambda *a: O.conv(*a, silu)[0], [x, w, b], i, dy))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(6, 6), (8, 4), (4, 0)])
def test_norm_rope_gradients(d, rot, interleaved):
    r = _rng(d + rot)
    x, w, dy = r.standard_normal((2, 3, 2, d)), r.standard_normal(d), r.standard_normal((2, 2, 3, d))
    angle = r.standard_normal((2, 3, rot // 2))
    how = np.cos(angle), np.sin(angle), 1e-3, interleaved
    grads = O.norm_rope_vjp(x, w, *how, dy)
    for i in range(2):
        _close(grads[i], _by_differences(lambda *a: O.norm_rope(*a, *how), [x, w], i, dy))


@pytest.mark.parametrize("softplus", [False, True])
@pytest.mark.parametrize("H,G", [(2, 1), (2, 2), (4, 2)])
def test_scan_gradients(H, G, softplus):
    r = _rng(H + G)
    B, n, P, N = 2, 4, 3, 2
    args = [r.standard_normal((B, n, H, P)), r.random((B, n, H)), -r.random(H), r.standard_normal((B, n, G, N)),
            r.standard_normal((B, n, G, N)), r.standard_normal(H), 0.1 * r.standard_normal(H)]
    dy = r.standard_normal((B, n, H, P))
    grads = O.ssm_vjp(*args, softplus, dy)
    for i in range(7):
        _close(grads[i], _by_differences(lambda *a: O.ssm(*a, softplus)[0], args, i, dy))


def test_absolute_sums_bound_the_gradients():
    r = _rng(5)
    args = [r.standard_normal((1, 6, 2, 3)), r.standard_normal((1, 6, 2)), -r.random(2), r.standard_normal((1, 6, 1, 4)),
            r.standard_normal((1, 6, 1, 4)), r.standard_normal(2), r.standard_normal(2)]
    dy = r.standard_normal((1, 6, 2, 3))
    for g, a in zip(O.ssm_vjp(*args, True, dy), O.ssm_vjp(*args, True, dy, absolute=True)):
        assert (np.abs(g) <= a * (1 + 1e-12)).all()


def test_planted_mistakes_show():
    """What the pins must catch: an exclusive state in the readout, a missing group sum."""
    r = _rng(9)
    x, dt, A = r.standard_normal((1, 5, 2, 3)), r.standard_normal((1, 5, 2)), -r.random(2)
    Bm, Cm = r.standard_normal((2, 1, 5, 1, 4))
    y, _ = O.ssm(x, dt, A, Bm, Cm)
    late, _ = O.ssm(x, dt, A, Bm, Cm * 0 + np.roll(Cm, 1, 1))
    assert np.abs(y - late).max() > 1e-3
    dy = r.standard_normal(x.shape)
    whole = O.ssm_vjp(x, dt, A, Bm, Cm, None, None, True, dy)[3]
    one = O.ssm_vjp(x[:, :, :1], dt[:, :, :1], A[:1], Bm, Cm, None, None, True, dy[:, :, :1])[3]
    assert np.abs(whole - one).max() > 1e-3
