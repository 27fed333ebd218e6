"""Gradients of the norms of a block: where the tokens do not fill a workgroup's
rows, without an eps that would hide what idle rows bring, against the oracle;
and weights wider than a launch.  Bars as in test_gpu_block.py: they hold for
any eps, since rows of these random values are far from zero."""
import pytest
import torch

import paper_2510_27258_amd as hla
from tests.test_gpu_block import TYPES, _gn_check, _rn_check, _rng, _say, _t

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


RN_SIZES = [(1, 5, 64), (2, 1, 20), (1, 33, 100), (1, 7, 200), (1, 1, 333), (3, 1021, 333), (1, 3, 1000), (1, 3, 2048),
            (1, 3, 9000)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", RN_SIZES)
def test_residual_norm_without_eps(size, types):
    for form in ("all", "weight", "scale", "no out", "no r"):
        _say(f"residual norm {size} {types} {form}")
        r = _rng(62, *size)
        x, y, gr, go = (_t(r.standard_normal(size), t) for t in (types[0], types[1], types[0], types[1]))
        w = _t(1 + 0.2 * r.standard_normal(size[-1]), types[1])
        post = None if form in ("weight", "scale") else _t(1 + 0.2 * r.standard_normal(size[-1]), types[1])
        scale = None if form == "weight" else _t(0.5 + 0.1 * r.standard_normal(size[-1]), types[1])
        go, gr = None if form == "no out" else go, None if form == "no r" else gr
        outs = hla.residual_norm_forward(x, y, w, post, scale, 0.5, 0.0)
        grads = hla.residual_norm_backward(x, y, w, post, scale, go, gr, 0.5, 0.0)
        assert all(torch.isfinite(t.float()).all() for t in (*outs, *grads) if t is not None)
        _rn_check(x, y, w, post, scale, 0.5, 0.0, go, gr, outs, grads, form)


@pytest.mark.parametrize("n", [1, 3])
def test_weights_of_many_groups(n):
    """A weight for each of 8193 groups of 8192: more columns than one launch sums, 64 threads a column of fewer than
    2^32.  Without a gate dweight is sum dout y / rms(y)."""
    G, d = 8193, 8192
    gen = torch.Generator("cuda").manual_seed(n)
    y, g = (torch.randn(1, n, G, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(G, d, generator=gen, device="cuda").bfloat16()
    _say(f"gated norm of {G} groups of {d}, {n} tokens")
    dy, _, dw = hla.gated_norm_backward(y, None, w, g, 1e-3)
    for at in (slice(0, 40), slice(4090, 4100), slice(G - 40, G)):
        yd, gd, wd = y[0, :, at].double(), g[0, :, at].double(), w[at].double()
        inv = (yd.square().mean(-1, keepdim=True) + 1e-3).rsqrt()
        hat = yd * inv
        ref = (gd * hat).sum(0)
        off = (dw[at].double() - ref).abs() - 2.0 ** -8 * (1 + 2.0 ** -7) * ref.abs() - 1e-5 * (gd * hat).abs().sum(0)
        assert off.max() <= 0
        gw = gd * wd
        ref = inv * (gw - hat * (gw * hat).mean(-1, keepdim=True))
        size = inv * (gw.abs() + hat.abs() * (gw * hat).abs().mean(-1, keepdim=True))
        off = (dy[0, :, at].double() - ref).abs() - 2.0 ** -8 * (1 + 2.0 ** -7) * ref.abs() - 1e-5 * size
        assert off.max() <= 0
