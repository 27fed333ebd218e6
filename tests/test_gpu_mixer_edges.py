"""The operators around the attention at the edges of their ranges: values
whose fp32 shortcuts fail, tensors at unusual addresses, infinities over many
segments.  Bars as in test_gpu_mixer.py where none is derived here."""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from oracle import mixer as O
from tests.test_gpu_mixer import (BF16, FP32, _check_scan, _conv_case, _n, _qk_case, _rng, _say, _ssm_case, _t, _tables,
                                  _within)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("big", [1e4, 1e5])
def test_tokens_behind_a_very_large_step(dtype, big):
    """One step of A dt = -1.6e5 or -1.6e6 in a tile: the running sum of the
    tile's decays is 2e6 in log2, whose fp32 neighbours are 0.25 apart, and the
    differences of the tokens behind it are a few tenths."""
    args, state, dy = _ssm_case(1, 150, 2, 32, 32, 1, dtype, 30, dt_dtype=FP32)
    x, dt, A, Bm, Cm, D, bias = args
    dt = 0.005 + 0.02 * torch.rand(dt.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    dt[0, 5, 0], dt[0, 70, 1] = big, big
    args = x, dt, torch.tensor([-16.0, -15.3], device="cuda"), Bm, Cm, D, None
    first = state.clone()
    y = hla.ssm_prefill(state, *args, softplus=False)
    _check_scan(args, first, y, state, False)


@pytest.mark.parametrize("K", [2, 4])
def test_fp32_silu_is_fp32_accurate(K):
    """A single tap of one, so that z is the input itself.  In units of 2^-23 of
    a value exp is off by one, a sum, a quotient and a product by a half each:
    s = 1 / (1 + exp(-z)) by 2 and y = z s by less than 4.  The slope s (1 + z
    (1 - s)) has 4 of its terms for s and the last three roundings, and s's own
    2, with half a rounding of 1 - s, times |z|."""
    z = torch.linspace(-80, 80, 64 * 1024, device="cuda").view(1, 1024, 64).contiguous()
    w = torch.zeros(64, K, device="cuda")
    w[:, K - 1] = 1
    zn = _n(z)
    s = 1 / (1 + np.exp(-zn))
    y = hla.conv_forward(z, w)
    _within(y, zn * s, np.abs(zn * s), 4 * 2 ** -23, "y")
    dx = hla.conv_backward(z, w, None, torch.ones_like(z))[0]
    _within(dx, s * (1 + zn * (1 - s)), s * (4 * (1 + np.abs(zn) * (1 - s)) + 3 * np.abs(zn) * s), 2 ** -23, "dx")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_qk_gradients_of_tiny_rows_without_eps(dtype):
    """Rows of 1e-14 with eps = 0: r is 1e14 and r^3 no fp32 number, dx is 1e14."""
    q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(2, 9, 3, 2, 64, 64, dtype, 31)
    q = (q.float() * 1e-14).to(dtype)
    grads = hla.qk_norm_rope_backward(q, k, qw, kw, cos, sin, pos, gq, gk, 0.0)
    c, s = (_n(t)[pos.cpu().numpy()] for t in (cos, sin))
    xn, wn, gn = _n(q), _n(qw), _n(gq)
    dx, dw = O.norm_rope_vjp(xn, wn, c, s, 0.0, False, gn)
    inv = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True))
    size = 2 * inv * (np.abs(gn).max(-1) * np.abs(wn).max()).transpose(0, 2, 1)[..., None]
    size = size * (1 + np.abs(xn * inv).max(-1, keepdims=True))
    if dtype == BF16:
        _within(grads[0], dx, np.abs(dx) + 1e-3 * size, 2 ** -8, "dx")
    else:
        _within(grads[0], dx, size, 1e-5, "dx")


def test_upstream_gradients_at_any_address():
    """The gradient of a slice of torch.cat is a contiguous view that starts
    where the slice does, here two bytes behind a boundary."""
    q = _qk_case(1, 20, 2, 2, 32, 32, BF16, 33)
    args, _, dy = _ssm_case(1, 80, 2, 32, 32, 1, BF16, 34)
    one = torch.ones(1, dtype=BF16, device="cuda")

    def grads(leaves, outs, ups, shift):
        flat = torch.cat([*([one] if shift else []), *(o.flatten() for o in outs)])
        up = torch.cat([*([one] if shift else []), *(u.flatten() for u in ups)])
        return torch.autograd.grad(flat, leaves, up)

    leaves = [t.clone().requires_grad_() for t in q[:4]]
    outs = hla.qk_norm_rope(*leaves, *q[4:7])
    for a, b in zip(grads(leaves, hla.qk_norm_rope(*leaves, *q[4:7]), q[7:9], True), grads(leaves, outs, q[7:9], False)):
        assert torch.equal(a, b)
    leaves = [t.clone().requires_grad_() for t in args]
    for a, b in zip(grads(leaves, [hla.ssm_scan(*leaves)], [dy], True), grads(leaves, [hla.ssm_scan(*leaves)], [dy], False)):
        assert torch.equal(a, b)


def test_attentions_upstream_gradient_at_any_address():
    """The same for the second-order attention, whose output is fp32."""
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v = (torch.randn(1, 2, 100, 64, generator=g, device="cuda").mul(0.1).to(BF16).requires_grad_() for _ in range(3))
    up = torch.randn(1, 2, 100, 64, generator=g, device="cuda")
    out = hla.hla2_attention(q, k, v)
    want = torch.autograd.grad(out, (q, k, v), up)
    flat = torch.cat([torch.zeros(1, device="cuda"), hla.hla2_attention(q, k, v).flatten()])
    got = torch.autograd.grad(flat, (q, k, v), torch.cat([torch.zeros(1, device="cuda"), up.flatten()]))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_step_of_more_heads_than_a_grid_dimension():
    """70400 heads: more than 65535."""
    args, state, _ = _ssm_case(2200, 1, 32, 16, 16, 1, BF16, 35)
    x, dt, A, Bm, Cm, D, bias = args
    first = state.clone()
    y = hla.ssm_step(state, x[:, 0], dt[:, 0], A, Bm[:, 0], Cm[:, 0], D, bias)
    _check_scan(args, first, y[:, None], state)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n", [700, 2100])
def test_infinities_over_segments(dtype, n):
    """Bad values in the first, a middle and the last segment, whose states the
    later segments take from the walk to the segments' ends (2 and 8 segments
    in bf16, 5 and 16 in fp32): what depends on them is infinite or NaN,
    whatever the segments, and the rest keeps its bits."""
    args, state, _ = _ssm_case(1, n, 2, 64, 64, 1, dtype, 36, views=False)
    clean_state = state.clone()
    clean = hla.ssm_prefill(clean_state, *args)
    for what in (0, 1, 3):
        for t in (3, n // 2, n - 2):
            for bad in (float("nan"), float("inf"), -float("inf")):
                if what == 1 and bad < 0:
                    continue                  # a step of softplus(-inf) = 0 is a number
                _say(f"n={n} {dtype} bad value {bad} in argument {what} at {t}")
                a = [m.clone() for m in args]
                st = state.clone()
                hit, hit_state = torch.zeros_like(clean, dtype=torch.bool), torch.zeros_like(st, dtype=torch.bool)
                if what == 0:
                    a[0][0, t, 1, 5] = bad
                    hit[0, t:, 1, 5] = hit_state[0, 1, :, 5] = True
                elif what == 1:
                    a[1][0, t, 1] = bad
                    hit[0, t:, 1] = hit_state[0, 1] = True
                else:
                    a[3][0, t, 0, 7] = bad
                    hit[0, t:] = hit_state[0, :, 7] = True
                y = hla.ssm_prefill(st, *a)
                assert torch.equal(~torch.isfinite(y), hit) and torch.equal(~torch.isfinite(st), hit_state)
                assert torch.equal(y[~hit], clean[~hit]) and torch.equal(st[~hit_state], clean_state[~hit_state])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_qk_tables_at_any_fp32_address(dtype):
    """Tables that start one float behind a 16-byte boundary."""
    q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(2, 30, 3, 2, 64, 64, dtype, 32)
    off = []
    for t in (cos, sin):
        flat = torch.empty(t.numel() + 1, device="cuda")
        flat[1:] = t.flatten()
        off.append(flat[1:].view_as(t))
        assert off[-1].data_ptr() % 16 == 4
    for f, more in ((hla.qk_norm_rope_forward, ()), (hla.qk_norm_rope_backward, (gq, gk))):
        for a, b in zip(f(q, k, qw, kw, cos, sin, pos, *more), f(q, k, qw, kw, *off, pos, *more)):
            assert torch.equal(a, b)
