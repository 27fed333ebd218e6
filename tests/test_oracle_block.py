"""Pins of the fp64 oracles of the operators of a block, without a GPU: closed
forms, and gradients against fp64 automatic differentiation of formulas written
a second time in torch, and against differences."""
import math

import numpy as np
import pytest
import torch

from oracle import block as O


def _rng(*seed):
    return np.random.default_rng(seed)


def _autograd(fn, args, ups):
    ts = [torch.from_numpy(a).requires_grad_() for a in args]
    outs = fn(*ts)
    outs = outs if isinstance(outs, tuple) else (outs,)
    return [g.numpy() for g in torch.autograd.grad(outs, ts, [torch.from_numpy(u) for u in ups])]


def _close(got, ref):
    for a, b in zip(got, ref):
        assert np.abs(a - b).max() <= 1e-11 * (1 + np.abs(b).max())


def _norm(v, eps):
    return v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_gated_norm(first, shared):
    r = _rng(1)
    y, z, g = (r.standard_normal((2, 3, 4, 5)) for _ in range(3))
    w = r.standard_normal((5,) if shared else (4, 5))

    def fn(y, z, w):
        gate = torch.nn.functional.silu(z)
        return _norm(y, 1e-2) * w * gate if first else _norm(y * gate, 1e-2) * w
    _close([O.gated_norm(y, z, w, 1e-2, first)], [fn(*map(torch.from_numpy, (y, z, w))).numpy()])
    _close(O.gated_norm_vjp(y, z, w, 1e-2, first, g), _autograd(fn, (y, z, w), [g]))


def test_gated_norm_of_constant_rows():
    y = np.full((1, 1, 1, 4), 3.0)
    assert np.allclose(O.gated_norm(y, eps=0.0), 1.0)
    assert np.allclose(O.gated_norm(y, z=np.zeros_like(y), eps=1.0), 0.0)
    assert np.allclose(O.gated_norm(y, eps=7.0), 3 / 4)          # sqrt(9 + 7) = 4


@pytest.mark.parametrize("post", [False, True])
def test_residual_norm(post):
    r = _rng(2)
    x, y, g, gr = (r.standard_normal((2, 3, 6)) for _ in range(4))
    w, p, s = (r.standard_normal(6) for _ in range(3))

    def fn(x, y, w, p, s):
        u = p * _norm(y, 1e-2) if post else y + 0 * p
        out = x + 0.5 * s * u
        return w * _norm(out, 1e-2), out
    args = (x, y, w, p if post else None, s)
    got = O.residual_norm_vjp(*args, 0.5, 1e-2, g, gr)
    ref = _autograd(fn, (x, y, w, p, s), [g, gr])
    _close([got[0], got[1], got[2], got[4]], [ref[0], ref[1], ref[2], ref[4]])
    if post:
        _close([got[3]], [ref[3]])


def test_recurrence_against_its_sum():
    """h_t as the sum of every earlier input times the decays between."""
    r = _rng(3)
    x, f, g = (r.standard_normal((2, 9, 3)) for _ in range(3))
    decay, fb, gb, state = r.standard_normal(3) - 2, r.standard_normal(3), r.standard_normal(3), r.standard_normal((2, 3))
    _, i, L, _, root = O.glr_gates(x, f, g, decay, fb, gb, 2.0)
    hs, last = O.glr(x, f, g, decay, fb, gb, 2.0, state)
    for t in range(9):
        ref = state * np.exp(L[:, :t + 1].sum(1))
        for s in range(t + 1):
            ref = ref + np.exp(L[:, s + 1:t + 1].sum(1)) * root[:, s] * i[:, s] * x[:, s]
        assert np.allclose(hs[:, t], ref, rtol=1e-12, atol=1e-13)
    assert np.array_equal(hs[:, -1], last)


def test_recurrence_gates_at_their_ends():
    one = np.ones((1, 1, 1))
    # a closed gate keeps the state and takes nothing; an open one with strong decay forgets it
    assert np.allclose(O.glr(one, -800 * one, one, np.zeros(1), state=5 * one[0])[1], 5)
    assert np.allclose(O.glr(one, 800 * one, 800 * one, np.full(1, 50.0), state=5 * one[0])[1], 1)


def test_recurrence_gradients():
    r = _rng(4)
    x, f, g, dy = (r.standard_normal((2, 7, 3)) for _ in range(4))
    decay, fb, gb = (r.standard_normal(3) for _ in range(3))

    def fn(x, f, g, decay, fb, gb):
        a = torch.exp(-3.0 * torch.nn.functional.softplus(decay) * torch.sigmoid(f + fb))
        b = torch.sqrt(1 - a * a) * torch.sigmoid(g + gb) * x
        h, hs = torch.zeros(2, 3, dtype=torch.float64), []
        for t in range(7):
            h = a[:, t] * h + b[:, t]
            hs.append(h)
        return torch.stack(hs, 1)
    args = (x, f, g, decay, fb, gb)
    _close(O.glr_vjp(*args, 3.0, dy), _autograd(fn, args, [dy]))
    for k in range(6):                        # and against differences
        step = 1e-6 * r.standard_normal(args[k].shape)
        up, down = ([a + s * step if j == k else a for j, a in enumerate(args)] for s in (1, -1))
        diff = ((O.glr(*up, 3.0)[0] - O.glr(*down, 3.0)[0]) * dy).sum() / 2
        assert abs(diff - (O.glr_vjp(*args, 3.0, dy)[k] * step).sum()) <= 1e-6 * abs(diff) + 1e-12


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_projections(kind):
    r = _rng(5)
    x, wg, wu, dh = r.standard_normal((2, 3, 4)), r.standard_normal((5, 4)), r.standard_normal((5, 4)), \
        r.standard_normal((2, 3, 5))

    def fn(x, wg, wu):
        return getattr(torch.nn.functional, kind)(x @ wg.T) * (x @ wu.T)
    _close([O.glu(x, wg, wu, kind)], [fn(*map(torch.from_numpy, (x, wg, wu))).numpy()])
    _close(O.glu_vjp(x, wg, wu, kind, dh)[:3], _autograd(fn, (x, wg, wu), [dh]))


def test_activations_by_hand():
    assert O.act(np.zeros(1), "silu")[1][0] == 0.5 and O.act(np.zeros(1), "gelu")[1][0] == 0.5
    assert math.isclose(O.act(np.ones(1), "gelu")[0][0], 0.8413447460685429)
    assert math.isclose(O.act(np.ones(1), "silu")[0][0], 1 / (1 + math.exp(-1)))
