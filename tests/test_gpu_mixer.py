"""The operators around the attention on the GPU against their fp64 oracles.

Bars, from the arithmetic:
  - A value rounded to bf16 (8 significant bits) is within 2^-8 of itself.
    fp32 sums of at most a few hundred terms stay within 1e-5 of the sum of
    their terms' absolute values.
  - The scan with bf16 inputs also rounds each score and the state it reads to
    bf16: 2^-8 of each term before the output's 2^-8, so y is held to 2^-7 of
    the same sum over absolute values; its state, and the fp32 gradients of the
    per-head parameters, to 1e-5 of theirs; the bf16 gradients to 2^-7.
"""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from oracle import mixer as O

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def _rng(*seed):
    return np.random.default_rng(seed)


def _t(x, dtype=FP32):
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(dtype).cuda()


def _n(x):
    return x.detach().double().cpu().numpy()


def _say(*a):
    print(*a, flush=True)


def _within(got, ref, scale, bar, what=""):
    got, ref = _n(got) if isinstance(got, torch.Tensor) else got, np.asarray(ref)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = np.abs(got - ref) - bar * scale
    assert (off <= 1e-30).all(), (what, float((np.abs(got - ref) / np.maximum(scale, 1e-30)).max()), bar)


# ----------------------------------------------------------------------------
# Convolution
def _conv_case(B, n, D, K, dtype, bias, seed):
    r = _rng(seed, B, n, D, K)
    x, w, dy = r.standard_normal((B, n, D)), r.standard_normal((D, K)) * 0.5, r.standard_normal((B, n, D))
    b = r.standard_normal(D) * 0.2 if bias else None
    st = r.standard_normal((B, K - 1, D))
    dev = [None if a is None else _t(a, dtype) for a in (x, w, b, dy, st)]
    return dev, [None if a is None else _n(a) for a in dev]


def _conv_scale(x, w, b, silu, st):
    """Sum of the terms' absolute values; SiLU's slope stays below 1.1."""
    return 1.1 * O.conv(np.abs(x), np.abs(w), None if b is None else np.abs(b), False, None if st is None else np.abs(st))[0]


SIZES = [(1, 1, 8), (2, 3, 64), (3, 17, 40), (2, 130, 333), (1, 257, 24), (5, 2, 1)]


@pytest.mark.parametrize("K,bias,silu", [(2, True, True), (3, False, False), (4, True, True), (4, False, True)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_conv_and_its_state(dtype, K, bias, silu):
    for B, n, D in SIZES:
        _say(f"conv B={B} n={n} D={D} K={K} {dtype}")
        (x, w, b, _, st), (xn, wn, bn, _, sn) = _conv_case(B, n, D, K, dtype, bias, 1)
        bar = 2 ** -8 if dtype == BF16 else 1e-5
        _within(hla.conv_forward(x, w, b, silu), O.conv(xn, wn, bn, silu)[0], _conv_scale(xn, wn, bn, silu, None), bar)
        y = hla.conv_prefill(st, x, w, b, silu)
        ref, _, last = O.conv(xn, wn, bn, silu, sn)
        _within(y, ref, _conv_scale(xn, wn, bn, silu, sn), bar)
        assert np.array_equal(_n(st), last)


@pytest.mark.parametrize("D", [64, 37])
def test_conv_pieces_and_steps_are_the_whole(D):
    """A prompt in pieces, then single tokens: the same sums, so the same bits."""
    (x, w, b, _, _), _ = _conv_case(2, 61, D, 4, BF16, True, 2)
    whole = hla.conv_forward(x, w, b)
    st = torch.zeros(2, 3, D, dtype=BF16, device="cuda")
    got, a = [], 0
    for p in (1, 2, 30, 3, 20):
        got.append(hla.conv_prefill(st, x[:, a:a + p], w, b))
        a += p
    got += [hla.conv_step(st, x[:, t], w, b)[:, None] for t in range(a, 61)]
    assert torch.equal(torch.cat(got, 1), whole)


@pytest.mark.parametrize("K,bias,silu", [(2, False, True), (3, True, True), (4, True, False), (4, True, True)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_conv_gradients(dtype, K, bias, silu):
    for B, n, D in SIZES + [(2, 1300, 136)]:
        _say(f"conv gradients B={B} n={n} D={D} K={K} {dtype}")
        (x, w, b, dy, _), (xn, wn, bn, dyn, _) = _conv_case(B, n, D, K, dtype, bias, 3)
        got = hla.conv_backward(x, w, b, dy, silu)
        ref = O.conv_vjp(xn, wn, bn, silu, dyn)
        scale = O.conv_vjp(np.abs(xn), np.abs(wn), None, False, np.abs(dyn))
        bar = 2 ** -8 if dtype == BF16 else 1e-5
        # z is a sum of K + 1 products in fp32 and the slope of SiLU changes by at most 0.5 of z's error
        for g, e, s in zip(got, ref, scale):
            if g is not None:
                _within(g, e, 1.1 * s, bar)


def test_conv_rows_of_a_wider_tensor_and_other_weights():
    """Slices of a projection (odd offsets included), broadcast rows, fp32 weights on bf16 inputs."""
    r = _rng(4)
    wide = _t(r.standard_normal((2, 50, 200)), BF16)
    w, b = _t(r.standard_normal((72, 4))), _t(r.standard_normal(72))
    for off in (0, 8, 3):
        x = wide[..., off:off + 72]
        same = hla.conv_forward(x.contiguous(), w, b)
        assert torch.equal(hla.conv_forward(x, w, b), same)
        got, want = hla.conv_backward(x, w, b, x), hla.conv_backward(x.contiguous(), w, b, x.contiguous())
        assert torch.equal(got[0], want[0])
        # the sums over the tokens are grouped by 16-byte rows or by single channels
        scale = O.conv_vjp(np.abs(_n(x)), np.abs(_n(w)), None, False, np.abs(_n(x)))
        for i in (1, 2):
            _within(got[i], _n(want[i]), 1.1 * scale[i], 1e-5)
    one = wide[:1, :1, :72].expand(2, 50, 72)
    assert torch.equal(hla.conv_forward(one, w, b), hla.conv_forward(one.contiguous(), w, b))


def test_conv_keeps_infinite_inputs_to_their_window():
    x = torch.ones(1, 40, 16, device="cuda", dtype=BF16)
    x[0, 10, 3], x[0, 20, 5] = float("nan"), float("inf")
    y = hla.conv_forward(x, torch.ones(16, 4, device="cuda"), None, False)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[0, 10:14, 3] = want[0, 20:24, 5] = True
    assert torch.equal(bad, want)


def test_conv_gradient_by_differences():
    """The fp32 kernel's gradient along a direction against differences of the
    kernel's own forward: a step of 2^-6 on a smooth function leaves a
    truncation of about 1e-4 of the slope, fp32 rounding 1e-5."""
    (x, w, b, dy, _), _ = _conv_case(2, 33, 20, 4, FP32, True, 5)
    grads = hla.conv_backward(x, w, b, dy)
    r = _rng(6)
    for i, a in enumerate((x, w, b)):
        v = _t(r.standard_normal(tuple(a.shape)))
        at = lambda e: (hla.conv_forward(*[q + e * v if j == i else q for j, q in enumerate((x, w, b))]).double() * dy).sum()  # noqa: E731
        slope = float((at(2 ** -6) - at(-2 ** -6)) / 2 ** -5)
        size = float((grads[i].double() ** 2).sum().sqrt() * (v.double() ** 2).sum().sqrt())
        assert abs(slope - float((grads[i].double() * v).sum())) <= 2e-3 * size


# ----------------------------------------------------------------------------
# Norm and rotation
def _tables(rot, count, scale=1.0):
    ang = np.arange(count)[:, None] * scale * 100.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
    return np.cos(ang), np.sin(ang)


def _qk_case(B, n, H, Hk, d, rot, dtype, seed, weights=True):
    r = _rng(seed, B, n, H, d)
    qkv = _t(r.standard_normal((B, n, (H + 2 * Hk) * d)) * 2, dtype)
    q, k = qkv[..., :H * d].unflatten(-1, (H, d)), qkv[..., H * d:(H + Hk) * d].unflatten(-1, (Hk, d))
    qw, kw = ((_t(1 + 0.2 * r.standard_normal(d), dtype) for _ in range(2)) if weights else (None, None))
    cos, sin = (_t(t) for t in _tables(rot, 4 * n + 10))
    pos = torch.from_numpy(r.integers(0, 4 * n + 10, (B, n))).cuda()
    gq, gk = (_t(r.standard_normal((B, h, n, d)), dtype) for h in (H, Hk))
    return q, k, qw, kw, cos, sin, pos, gq, gk


QK = [(1, 1, 1, 1, 16, 16), (2, 7, 4, 2, 64, 64), (2, 5, 3, 3, 128, 128), (1, 9, 6, 1, 80, 40), (3, 4, 2, 2, 96, 48),
      (1, 3, 2, 1, 256, 256), (2, 3, 8, 4, 128, 0), (1, 70, 5, 5, 24, 20), (4, 300, 8, 8, 128, 64)]


def _qk_scale(ref):
    """An output element is two products of a normed row."""
    return np.abs(ref).max(-1, keepdims=True) + 0 * ref


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_qk_norm_rope_and_gradients(dtype, interleaved):
    for case in QK:
        B, n, H, Hk, d, rot = case
        _say(f"qk norm rope {case} {dtype} interleaved={interleaved}")
        q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(*case, dtype, 1)
        outs = hla.qk_norm_rope_forward(q, k, qw, kw, cos, sin, pos, 1e-3, interleaved)
        grads = hla.qk_norm_rope_backward(q, k, qw, kw, cos, sin, pos, gq, gk, 1e-3, interleaved)
        c, s = (_n(t)[pos.cpu().numpy()] for t in (cos, sin))
        bar = 2 ** -8 if dtype == BF16 else 1e-5
        for i, (x, w, g) in enumerate(((q, qw, gq), (k, kw, gk))):
            xn, wn, gn = _n(x), _n(w), _n(g)
            ref = O.norm_rope(xn, wn, c, s, 1e-3, interleaved)
            _within(outs[i], ref, _qk_scale(ref), bar, "out")
            assert outs[i].is_contiguous()
            dx, dw = O.norm_rope_vjp(xn, wn, c, s, 1e-3, interleaved, gn)
            # dx is a difference of two terms of the size of r g w, g of two products
            inv = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True) + 1e-3)
            size = (inv * (np.abs(gn).max(-1) * np.abs(wn).max()).transpose(0, 2, 1)[..., None]) * 2
            size = size * (1 + np.abs(xn * inv).max(-1, keepdims=True))
            _within(grads[i], dx, np.abs(dx) if dtype == BF16 else size, bar, "dx") if dtype == FP32 else _within(
                grads[i], dx, np.abs(dx) + 1e-3 * size, bar, "dx")
            # sums over all rows: of |g xhat| terms
            rows = np.abs(gn).max(-1)[..., None] * np.abs(xn * inv).transpose(0, 2, 1, 3) * 2
            _within(grads[2 + i], dw, np.abs(dw) * (bar if dtype == BF16 else 0) / 1e-5 + rows.sum((0, 1, 2)), 1e-5, "dw")


def test_qk_without_weights_positions_or_rotation():
    q, k, _, _, cos, sin, _, _, _ = _qk_case(2, 6, 2, 2, 64, 64, BF16, 2, weights=False)
    a = hla.qk_norm_rope_forward(q, k, None, None, cos, sin)
    one = torch.ones(64, device="cuda")
    pos = torch.arange(6, device="cuda")
    for p in (pos, pos.int(), pos.expand(2, 6)):
        for x, y in zip(a, hla.qk_norm_rope_forward(q, k, one, one, cos, sin, p)):
            assert torch.equal(x, y)
    bare = hla.qk_norm_rope_forward(q, k, one * 64 ** -0.5, None)
    assert torch.allclose(bare[0].float().norm(dim=-1), torch.ones(2, 2, 6, device="cuda"), atol=4e-3)
    # unit weights and none have the same rows; a weight on one side leaves the other's gradient out
    grads = hla.qk_norm_rope_backward(q, k, one, None, cos, sin, None, a[0], a[1])
    assert grads[2].shape == (64,) and grads[3] is None


def test_positions_outside_the_tables_give_nan():
    q, k, qw, kw, cos, sin, _, gq, gk = _qk_case(1, 4, 2, 1, 64, 32, FP32, 3)
    pos = torch.tensor([[0, -1, cos.shape[0], cos.shape[0] - 1]], device="cuda")
    for y in hla.qk_norm_rope_forward(q, k, qw, kw, cos, sin, pos):
        assert torch.isnan(y[:, :, 1:3, :32]).all() and torch.isfinite(y[:, :, 1:3, 32:]).all()
        assert torch.isfinite(y[:, :, [0, 3]]).all()
    dq = hla.qk_norm_rope_backward(q, k, qw, kw, cos, sin, pos, gq, gk)[0]
    assert torch.isfinite(dq[:, [0, 3]]).all() and torch.isnan(dq[:, 1:3]).any()


def test_qk_rows_of_zeros_and_of_infinities():
    """A row of zeros stays zero (eps > 0); an infinite element spoils its own row alone."""
    q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(1, 5, 3, 3, 64, 64, BF16, 4)
    q, k = q.clone(), k.clone()
    q[0, 1, 2], k[0, 3, 0, 7] = 0, float("inf")
    qo, ko = hla.qk_norm_rope_forward(q, k, qw, kw, cos, sin, pos)
    assert (qo[0, 2, 1] == 0).all() and torch.isfinite(qo).all()
    bad = ~torch.isfinite(ko).all(-1)
    assert bad[0, 0, 3] and bad.sum() == 1
    assert torch.isfinite(hla.qk_norm_rope_backward(q, q, qw, kw, cos, sin, pos, gq, gk)[0]).all()


def test_qk_gradient_by_differences():
    q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(2, 5, 3, 2, 48, 32, FP32, 5)
    grads = hla.qk_norm_rope_backward(q, k, qw, kw, cos, sin, pos, gq, gk)
    r = _rng(8)
    args = [q, k, qw, kw]
    for i in range(4):
        v = _t(r.standard_normal(tuple(args[i].shape)))

        def at(e):
            moved = [a + e * v if j == i else a for j, a in enumerate(args)]
            return sum(float((o.double() * g).sum()) for o, g in
                       zip(hla.qk_norm_rope_forward(*moved, cos, sin, pos), (gq, gk)))
        slope = (at(2 ** -6) - at(-2 ** -6)) / 2 ** -5
        size = float((grads[i].double() ** 2).sum().sqrt() * (v.double() ** 2).sum().sqrt())
        assert abs(slope - float((grads[i].double() * v).sum())) <= 2e-3 * size


# ----------------------------------------------------------------------------
# State space scan
def _ssm_case(B, n, H, P, N, G, dtype, seed, dt_dtype=None, views=True):
    r = _rng(seed, B, n, H, P, N)
    xbc = _t(r.standard_normal((B, n, H * P + 2 * G * N)), dtype)
    x = xbc[..., :H * P].unflatten(-1, (H, P))
    Bm = xbc[..., H * P:H * P + G * N].unflatten(-1, (G, N))
    Cm = xbc[..., H * P + G * N:].unflatten(-1, (G, N))
    if not views:
        x, Bm, Cm = x.contiguous(), Bm.contiguous(), Cm.contiguous()
    dt = _t(r.standard_normal((B, n, H)), dt_dtype or dtype)
    A, D, bias = _t(-0.2 - 8 * r.random(H)), _t(r.standard_normal(H)), _t(r.standard_normal(H) - 3)
    state = _t(r.standard_normal((B, H, N, P)))
    dy = _t(r.standard_normal((B, n, H, P)), dtype)
    return (x, dt, A, Bm, Cm, D, bias), state, dy


def _abs(args):
    x, dt, A, Bm, Cm, D, bias = args
    return np.abs(x), dt, A, np.abs(Bm), np.abs(Cm), None if D is None else np.abs(D), bias


def _check_scan(args, state, got, got_state, softplus=True):
    an = [None if a is None else _n(a) for a in args]
    sn = None if state is None else _n(state)
    ref, last = O.ssm(*an, softplus, sn)
    scale, slast = O.ssm(*_abs(an), softplus, None if sn is None else np.abs(sn))
    _within(got, ref, scale, 2 ** -7 if args[0].dtype == BF16 else 1e-5, "y")
    if got_state is not None:
        _within(got_state, last, slast, 1e-5, "state")


SSM = [(1, 1, 1, 16, 16, 1), (2, 2, 2, 64, 64, 1), (1, 31, 4, 32, 16, 2), (2, 63, 2, 64, 128, 2), (1, 64, 3, 128, 32, 1),
       (1, 65, 2, 48, 80, 1), (2, 130, 4, 112, 48, 4), (1, 300, 2, 128, 128, 1), (1, 700, 2, 16, 64, 2)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", SSM)
def test_scan_and_its_state(case, dtype):
    B, n, H, P, N, G = case
    _say(f"scan {case} {dtype}")
    args, state, _ = _ssm_case(*case, dtype, 1)
    _check_scan(args, None, hla.ssm_forward(*args), None)
    first = state.clone()
    y = hla.ssm_prefill(state, *args)
    _check_scan(args, first, y, state)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scan_without_skip_bias_or_softplus(dtype):
    args, state, _ = _ssm_case(2, 90, 2, 32, 32, 1, dtype, 2, dt_dtype=FP32)
    x, dt, A, Bm, Cm, D, bias = args
    dt = dt.abs() * 0.1
    for a, soft in (((x, dt, A, Bm, Cm, None, None), False), ((x, dt, A, Bm, Cm, D, None), True),
                    ((x, dt - 5, A, Bm, Cm, None, bias), True)):
        st = state.clone()
        y = hla.ssm_prefill(st, *a, softplus=soft)
        _check_scan(a, state, y, st, soft)


@pytest.mark.parametrize("B,H", [(1, 1), (2, 3), (40, 14)])
def test_scan_over_segments(B, H):
    """Long heads cut into many segments (one head: as many as there are), a
    few, and none (560 heads)."""
    args, state, _ = _ssm_case(B, 2100 if B < 40 else 130, H, 32, 32, 1, BF16, 3)
    first = state.clone()
    y = hla.ssm_prefill(state, *args)
    _check_scan(args, first, y, state)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prompt_in_pieces_then_steps(dtype):
    """Pieces of one token, of part of a tile, of many tiles, then single tokens."""
    args, state, _ = _ssm_case(2, 500, 4, 64, 64, 2, dtype, 4)
    x, dt, A, Bm, Cm, D, bias = args
    first, got, a = state.clone(), [], 0
    for p in (1, 63, 70, 350):
        cut = slice(a, a + p)
        got.append(hla.ssm_prefill(state, x[:, cut], dt[:, cut], A, Bm[:, cut], Cm[:, cut], D, bias))
        a += p
    for t in range(a, 500):
        got.append(hla.ssm_step(state, x[:, t], dt[:, t], A, Bm[:, t], Cm[:, t], D, bias)[:, None])
    _check_scan(args, first, torch.cat(got, 1), state)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_step_sizes(dtype):
    for case in [(1, 1, 1, 16, 16, 1), (3, 1, 4, 64, 128, 2), (2, 1, 3, 48, 80, 1), (2, 1, 2, 128, 128, 1),
                 (1, 1, 2, 112, 96, 2)]:
        _say(f"step {case} {dtype}")
        args, state, _ = _ssm_case(*case, dtype, 5)
        first = state.clone()
        x, dt, A, Bm, Cm, D, bias = args
        y = hla.ssm_step(state, x[:, 0], dt[:, 0], A, Bm[:, 0], Cm[:, 0], D, bias)
        _check_scan(args, first, y[:, None], state)


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("case", SSM)
def test_scan_gradients(case, softplus):
    _say(f"scan gradients {case} softplus={softplus}")
    args, _, dy = _ssm_case(*case, BF16, 6)
    args = list(args)
    if not softplus:
        args[1], args[6] = args[1].abs() * 0.1, args[6] * 0
    got = hla.ssm_backward(*args, dy, softplus)
    an, dn = [_n(a) for a in args], _n(dy)
    ref = O.ssm_vjp(*an, softplus, dn)
    scale = O.ssm_vjp(*an, softplus, dn, absolute=True)
    for name, g, e, s in zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dbias"), got, ref, scale):
        if name in ("dx", "dB", "dC"):
            _within(g, e, s, 2 ** -7, name)
        elif name == "ddt":
            _within(g, e, np.abs(e) + (1e-5 * 2 ** 8) * s, 2 ** -8, name)
        else:
            _within(g, e, s, 1e-5, name)


def test_scan_gradients_over_segments_and_subsets():
    """Many segments a head and several head subsets a group, against autograd's
    sum over groups: shared B and C get the sum of their heads' gradients."""
    args, _, dy = _ssm_case(1, 1100, 6, 32, 32, 1, BF16, 7, dt_dtype=FP32)
    got = hla.ssm_backward(*args, dy)
    x, dt, A, Bm, Cm, D, bias = args
    parts = [hla.ssm_backward(x[:, :, h:h + 1].contiguous(), dt[:, :, h:h + 1].contiguous(), A[h:h + 1], Bm, Cm, D[h:h + 1],
                              bias[h:h + 1], dy[:, :, h:h + 1].contiguous()) for h in range(6)]
    assert torch.allclose(got[1], torch.cat([p[1] for p in parts], 2), rtol=1e-4, atol=1e-5)
    for i in (3, 4):
        total = sum(p[i].double() for p in parts)
        size = sum(p[i].double().abs() for p in parts)
        assert ((got[i].double() - total).abs() <= 2 ** -7 * size + 1e-6).all()


def test_scan_gradient_by_differences():
    """Along a direction: differences of the fp32 kernel's forward on the bf16
    values (a step of 2^-6) against the bf16 kernel's gradient, whose elements
    are rounded to 2^-8 of themselves."""
    args, _, dy = _ssm_case(1, 150, 2, 32, 32, 1, BF16, 8)
    grads = hla.ssm_backward(*args, dy)
    wide = [a.float() for a in args]
    r = _rng(9)
    for i in range(7):
        v = _t(r.standard_normal(tuple(wide[i].shape)))

        def at(e):
            moved = [(a + e * v if j == i else a) for j, a in enumerate(wide)]
            return float((hla.ssm_forward(*moved).double() * dy).sum())
        slope = (at(2 ** -6) - at(-2 ** -6)) / 2 ** -5
        size = float((grads[i].double() ** 2).sum().sqrt() * (v.double() ** 2).sum().sqrt())
        assert abs(slope - float((grads[i].double() * v).sum())) <= 4e-3 * size, i


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_later_infinities_do_not_reach_earlier_tokens(dtype):
    """NaN and infinities in x, B, C and dt: the outputs before them keep their
    bits, the ones that depend on them are not finite, and so is the state's
    column (x), row (B) or all of it (dt)."""
    args, state, _ = _ssm_case(1, 200, 2, 64, 64, 1, dtype, 10, views=False)
    first = state.clone()
    clean_state = state.clone()
    clean = hla.ssm_prefill(clean_state, *args)
    for what, t in ((0, 70), (3, 70), (4, 70), (1, 70), (0, 63), (3, 199), (0, 0)):
        for bad in (float("nan"), float("inf")):
            a = [m.clone() for m in args]
            if what in (0, 1):
                a[what][0, t, 1] = bad if what == 1 else a[what][0, t, 1]
                if what == 0:
                    a[0][0, t, 1, 5] = bad
            else:
                a[what][0, t, 0, 7] = bad
            st = first.clone()
            y = hla.ssm_prefill(st, *a)
            _say(f"bad value {bad} in argument {what} at {t}")
            hit = torch.zeros_like(y, dtype=torch.bool)
            hit_state = torch.zeros_like(st, dtype=torch.bool)
            if what == 0:
                hit[0, t:, 1, 5] = hit_state[0, 1, :, 5] = True
            elif what == 1:
                hit[0, t:, 1] = hit_state[0, 1] = True
            elif what == 3:
                hit[0, t:], hit_state[0, :, 7] = True, True
            else:
                hit[0, t] = True
            assert torch.equal(~torch.isfinite(y), hit) and torch.equal(~torch.isfinite(st), hit_state)
            assert torch.equal(y[~hit], clean[~hit]) and torch.equal(st[~hit_state], clean_state[~hit_state])


def test_steep_and_still_heads():
    """Decays that underflow at once (A dt = -2000) and none at all (A = 0)."""
    args, state, _ = _ssm_case(1, 130, 2, 32, 32, 1, BF16, 11)
    x, dt, A, Bm, Cm, D, bias = args
    A = torch.tensor([-2000.0, 0.0], device="cuda")
    args = (x, dt, A, Bm, Cm, D, torch.zeros_like(bias))
    first = state.clone()
    y = hla.ssm_prefill(state, *args)
    _check_scan(args, first, y, state)
    grads = hla.ssm_backward(*args, y)
    assert all(torch.isfinite(g).all() for g in grads)


# ----------------------------------------------------------------------------
# All of them
def _calls():
    c, _ = _conv_case(2, 200, 64, 4, BF16, True, 20)
    q = _qk_case(2, 100, 4, 2, 64, 64, BF16, 21)
    s, state, dy = _ssm_case(2, 400, 4, 64, 64, 2, BF16, 22)
    return {
        "conv": lambda: [hla.conv_forward(*c[:3])],
        "conv gradients": lambda: hla.conv_backward(*c[:4]),
        "qk": lambda: hla.qk_norm_rope_forward(*q[:7]),
        "qk gradients": lambda: hla.qk_norm_rope_backward(*q),
        "scan": lambda: [hla.ssm_forward(*s)],
        "scan gradients": lambda: hla.ssm_backward(*s, dy),
        "prompt": lambda: [hla.ssm_prefill(state.clone(), *s)],
    }


def test_same_inputs_give_the_same_bits():
    for name, f in _calls().items():
        _say(name)
        for a, b in zip(f(), f()):
            assert torch.equal(a, b), name


def test_another_stream_and_a_captured_graph():
    for name, f in _calls().items():
        _say(name)
        want = [x.clone() for x in f()]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = f()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = f()
        for _ in range(3):
            for x in held:
                x.fill_(7)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want)), name


def test_a_captured_graph_of_the_widest_scan():
    """P = N = 128 takes more than 64 KB of LDS a workgroup, which a launch has to ask for."""
    s, state, dy = _ssm_case(1, 300, 2, 128, 128, 1, BF16, 26)
    for f in (lambda: [hla.ssm_forward(*s)], lambda: hla.ssm_backward(*s, dy), lambda: [hla.ssm_prefill(state.clone(), *s)]):
        want = [x.clone() for x in f()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = f()
        for _ in range(3):
            for x in held:
                x.fill_(7)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_autograd_ops_give_the_kernels_gradients():
    c, _ = _conv_case(2, 50, 24, 3, BF16, True, 23)
    leaves = [t.clone().requires_grad_() for t in c[:3]]
    hla.short_conv(*leaves).backward(c[3])
    for a, b in zip(leaves, hla.conv_backward(*c[:4])):
        assert torch.equal(a.grad, b)
    q = _qk_case(1, 20, 2, 2, 32, 32, FP32, 24)
    leaves = [t.clone().requires_grad_() for t in q[:4]]
    qo, ko = hla.qk_norm_rope(*leaves, *q[4:7])
    torch.autograd.backward([qo.transpose(1, 2), ko], [q[7].transpose(1, 2), q[8]])
    for a, b in zip(leaves, hla.qk_norm_rope_backward(*q)):
        assert torch.equal(a.grad, b)
    s, _, dy = _ssm_case(1, 80, 2, 32, 32, 1, BF16, 25)
    leaves = [t.clone().requires_grad_() for t in s]
    hla.ssm_scan(*leaves).backward(dy)
    for a, b in zip(leaves, hla.ssm_backward(*s, dy)):
        assert torch.equal(a.grad, b)
    # broadcast upstream gradients: the sum's
    y = hla.short_conv(c[0].requires_grad_(), c[1], c[2])
    y.sum().backward()
    ones = hla.conv_backward(c[0], c[1], c[2], torch.ones_like(y))
    assert torch.equal(c[0].grad, ones[0])


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 bytes and 2^31 elements: the last rows against
    the same rows by themselves."""
    n, D = 270000, 8192
    x = torch.empty(1, n, D, dtype=BF16, device="cuda")
    x.normal_(generator=torch.Generator("cuda").manual_seed(1))
    w = torch.randn(D, 4, device="cuda")
    _say("conv")
    y = hla.conv_forward(x, w)
    st = x[:, -1003:-1000].clone()
    assert torch.equal(y[:, -1000:], hla.conv_prefill(st, x[:, -1000:], w))
    _say("norm and rotation")
    q = x.unflatten(-1, (64, 128))
    cos, sin = (_t(t) for t in _tables(128, 1000))
    pos = torch.arange(n, device="cuda")[None] % 1000
    qo, _ = hla.qk_norm_rope_forward(q, q[:, :, :1], None, None, cos, sin, pos)
    tail, _ = hla.qk_norm_rope_forward(q[:, -100:], q[:, -100:, :1], None, None, cos, sin, pos[:, -100:])
    assert torch.equal(qo[:, :, -100:], tail)
    del qo, tail, y
    _say("scan")
    Bm = torch.randn(1, n, 1, 16, dtype=BF16, device="cuda")
    dt = torch.randn(1, n, 64, dtype=BF16, device="cuda")
    A = -torch.rand(64, device="cuda")
    y = hla.ssm_forward(q, dt, A, Bm, Bm)
    state = torch.zeros(1, 64, 16, 128, device="cuda")
    cut = n - 1000
    hla.ssm_prefill(state, q[:, cut - 4000:cut], dt[:, cut - 4000:cut], A, Bm[:, cut - 4000:cut], Bm[:, cut - 4000:cut])
    tail = hla.ssm_prefill(state, q[:, cut:], dt[:, cut:], A, Bm[:, cut:], Bm[:, cut:])
    keep = A < -0.1                      # heads that forget what is 4000 tokens back
    a, b = y[:, cut:][:, :, keep].float(), tail[:, :, keep].float()
    assert (a - b).abs().max() <= 2 ** -6 * a.abs().max()
