"""The fp64 oracle of GELU far below zero, against Laplace's continued fraction
of the normal distribution's tail: Q(x) = phi(x) / (x + 1 / (x + 2 / (x + ...))).
From x = 3 on 400 levels of it have settled to 1e-12 of itself, which the test
checks; the complementary error function is good to a few 2^-53 of itself, and
its argument's rounding, of x sqrt(1/2), moves it by at most x^2 2^-52 < 1e-13."""
import math

import numpy as np

from oracle import block as O


def _tail(x, levels):
    f = x
    for k in range(levels, 0, -1):
        f = x + k / f
    return np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi) / f


def test_gelu_far_below_zero():
    x = np.linspace(3, 20, 171)
    q = _tail(x, 400)
    assert (np.abs(_tail(x, 800) / q - 1) <= 1e-12).all()
    f, d = O.act(-x, "gelu")
    assert (np.abs(f / (-x * q) - 1) <= 1e-11).all()
    slope = q - x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    assert (np.abs(d / slope - 1) <= 1e-11).all()
