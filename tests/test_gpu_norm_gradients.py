"""Gradients of the norms of a block where the tokens do not fill a workgroup's
rows, without an eps that would hide what idle rows bring, against the oracle.
Bars as in test_gpu_block.py: they hold for any eps, since rows of these random
values are far from zero."""
import pytest
import torch

import paper_2510_27258_amd as hla
from tests.test_gpu_block import TYPES, _gn_check, _rng, _say, _t

pytestmark = pytest.mark.gpu

# B, n, G, d: 32, 16, 8 and 4 rows a workgroup, never a multiple of them
GN_SIZES = [(1, 5, 1, 64), (1, 33, 1, 64), (1, 3, 3, 64), (2, 5, 7, 20), (1, 2, 1, 100), (1, 7, 1, 200), (1, 1, 1, 333),
            (3, 1021, 1, 333), (1, 3, 1, 1000), (1, 2, 2, 2048), (1, 3, 1, 9000)]


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", GN_SIZES)
def test_gated_norm_without_eps(size, types, first):
    B, n, G, d = size
    for form in ("shared", "per group", "no gate"):
        _say(f"gated norm {size} {types} first={first} {form}")
        r = _rng(61, *size)
        y = _t(r.standard_normal(size), types[0])
        z = None if form == "no gate" else _t(r.standard_normal(size), types[1])
        w = _t(1 + 0.2 * r.standard_normal((G, d) if form == "per group" else d), types[1])
        g = _t(r.standard_normal(size), types[1])
        out = hla.gated_norm_forward(y, z, w, 0.0, first, types[1])
        grads = hla.gated_norm_backward(y, z, w, g, 0.0, first)
        assert all(torch.isfinite(t.float()).all() for t in (out, *grads) if t is not None)
        _gn_check(y, z, w, 0.0, first, g, out, grads, form)
