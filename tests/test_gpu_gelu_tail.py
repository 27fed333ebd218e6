"""GELU of the gated projections far below zero, by relative error: there the
normal distribution is a small number of its own, not a difference from one.

Bars, from the arithmetic.  The pre-activations are the inputs themselves (each
a bf16 times one, beside zeros), so p is exact, and so is u = 1.  The
distribution's tail is e^(-x^2) times a function of x, x^2 = p^2 / 2: rounding x
moves it by 2 x^2 2^-24, rounding x^2 and its product with log2 e by x^2 2^-24
each, at most x^2 = 72 here, and the function's steps by less than 20 2^-24:
(4 72 + 20) 2^-24 < 2^-15.  Outputs are rounded to bf16 once, 2^-8; dp and du
are rounded before the products that bring them out, which are exact (one term
beside zeros), and the result then is a bf16 already."""
import math

import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from tests.test_gpu_block import BF16, _n, _say

pytestmark = pytest.mark.gpu

ROUNDED = 2.0 ** -8 * (1 + 2.0 ** -7)
TAIL = 2.0 ** -15
_erfc = np.vectorize(math.erfc, otypes=[float])


def _case(p):
    """Tokens of pre-activation p and linear part 1, each with a column of x of its own."""
    n, F = p.numel(), 24
    x = torch.zeros(1, n, -(-(n + 1) // 8) * 8, device="cuda", dtype=BF16)
    x[0, :, 0] = p
    x[0, torch.arange(n), 1 + torch.arange(n)] = 1.0
    wg, wu = torch.zeros(F, x.shape[-1], device="cuda", dtype=BF16), torch.zeros(F, x.shape[-1], device="cuda", dtype=BF16)
    wg[:, 0] = 1.0
    wu[:, 1:] = 1.0
    return x, wg, wu


# up to 16 tokens take a kernel of their own, 73 and 600 the tiles
@pytest.mark.parametrize("n", [1, 10, 73, 600])
def test_relative_error_of_the_tail(n):
    p = torch.linspace(-12, -3, n, device="cuda").to(BF16)
    x, wg, wu = _case(p)
    pn = _n(p)
    below, density = 0.5 * _erfc(-pn / math.sqrt(2)), np.exp(-0.5 * pn * pn) / math.sqrt(2 * math.pi)
    _say(f"tail of {n} tokens")
    h = _n(hla.glu_forward(x, wg, wu, "gelu"))[0]
    ref = (pn * below)[:, None]
    assert (np.abs(h - ref) <= (ROUNDED + TAIL) * np.abs(ref)).all(), np.abs(h / ref - 1).max()
    dh = torch.full((1, n, wg.shape[0]), 1.5, device="cuda", dtype=BF16)
    _, dwg, dwu = (_n(t) for t in hla.glu_backward(x, wg, wu, dh, "gelu"))
    own = 1 + np.arange(n)
    ref = 1.5 * pn * below
    assert (np.abs(dwu[:, own] - ref) <= (ROUNDED + TAIL) * np.abs(ref)).all(), np.abs(dwu[:, own] / ref - 1).max()
    ref, size = 1.5 * (below + pn * density), 1.5 * (below + np.abs(pn) * density)
    assert (np.abs(dwg[:, own] - ref) <= ROUNDED * np.abs(ref) + TAIL * size).all()


def test_both_sides_of_zero():
    """The two branches, and zero: the whole activation against the formula."""
    p = torch.cat([torch.linspace(-4, 4, 201, device="cuda"), torch.zeros(1, device="cuda")]).to(BF16)
    x, wg, wu = _case(p)
    pn = _n(p)
    ref = (pn * 0.5 * _erfc(-pn / math.sqrt(2)))[:, None]
    h = _n(hla.glu_forward(x, wg, wu, "gelu"))[0]
    assert (np.abs(h - ref) <= (ROUNDED + TAIL) * np.abs(ref)).all()
