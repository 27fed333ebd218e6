"""The operators of a block on the GPU against their fp64 oracles.

Bars, from the arithmetic:
  - A value rounded to bf16 is within 2^-8 of itself.  fp32 sums of a few
    hundred terms, or of thousands in lanes that join, stay within 1e-5 of the
    sum of their terms' absolute values, and so do the few fp32 steps around
    them; a sum whose terms are such sums is held to the sum of their scales.
    The sigmoid of bf16 inputs is within 2^-16.
  - The recurrence multiplies up to n decays, each with two steps of 2^-24, and
    forms each by some 40 steps: (n + 64) 2^-23 of its sum over absolute values,
    and twice that for gradients, which multiply two such sums.
  - The projections' sums are within 1e-5 of their sums over absolute values;
    both activations' slopes are below 1.13, their second derivatives below 1.
    The gradients of the projections are rounded to bf16 before their products:
    2^-8 of each term, and 2^-8 of the result.  Such roundings are even over
    their range: the whole result is within sqrt(2) 2^-8 / sqrt(3) in the 2-norm.
"""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from oracle import block as O

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
FINE = 1e-5


def _rng(*seed):
    return np.random.default_rng(seed)


def _t(x, dtype=FP32):
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(dtype).cuda()


def _n(x):
    return None if x is None else x.detach().double().cpu().numpy()


def _say(*a):
    print(*a, flush=True)


def _within(got, ref, scale, bar=FINE, what=""):
    """|got - ref| <= bar scale, and the rounding of got's type."""
    step = 2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24
    got, ref = _n(got), np.asarray(ref)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = np.abs(got - ref) - step * np.abs(ref) * (1 + 2.0 ** -7) - bar * scale
    assert (off <= 1e-30).all(), (what, float(off.max()), float((np.abs(got - ref) / np.maximum(scale, 1e-30)).max()), bar)


# ----------------------------------------------------------------------------
TYPES = [(BF16, BF16), (FP32, FP32), (FP32, BF16)]
GN_SIZES = [(1, 1, 1, 8), (2, 3, 4, 64), (1, 5, 7, 80), (3, 9, 2, 128), (2, 33, 3, 16), (1, 4, 5, 33), (2, 3, 1, 1000),
            (1, 7, 2, 2048), (1, 3, 1, 5000), (2, 2, 1, 16384), (1, 2, 33, 1), (1, 3, 300, 24), (1, 2, 1, 11111)]


def _gn_check(y, z, w, eps, first, gout, out, grads, what):
    yn, zn, wn, gn = map(_n, (y, z, w, gout))
    ref = O.gated_norm(yn, zn, wn, eps, first)
    _within(out, ref, np.abs(ref), what=what)
    dy, dz, dw = O.gated_norm_vjp(yn, zn, wn, eps, first, gn)
    w1 = 1.0 if wn is None else np.abs(wn)
    s = None if zn is None else O.sigmoid(zn)
    gate = 1.0 if zn is None else np.abs(zn * s)
    v = np.abs(yn) * (1.0 if first else gate)
    inv = O.inverse_rms(v, eps)
    gh = np.abs(gn) * (gate if first else 1.0)
    dv = inv * (gh * w1 + v * inv * (gh * w1 * v * inv).mean(-1, keepdims=True))
    _within(grads[0], dy, dv * (1.0 if first else gate), what=what + " dy")
    if zn is not None:
        slope = s * (1 + np.abs(zn) * (1 - s))
        _within(grads[1], dz, (np.abs(gn) * w1 * v * inv if first else dv * np.abs(yn)) * slope, what=what + " dz")
    if wn is not None:
        terms = gh * v * inv
        _within(grads[2], dw, terms.sum((0, 1) if wn.ndim == 2 else (0, 1, 2)), what=what + " dw")


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", GN_SIZES)
def test_gated_norm(size, types, first):
    B, n, G, d = size
    for form in ("shared", "per group", "no gate", "no weight", "heads first"):
        _say(f"gated norm {size} {types} first={first} {form}")
        r = _rng(1, *size)
        y = _t(r.standard_normal((B, G, n, d) if form == "heads first" else (B, n, G, d)), types[0])
        if form == "heads first":
            y = y.transpose(1, 2)
        z = None if form == "no gate" else _t(r.standard_normal((B, n, 2 * G * d)), types[1])[..., G * d:].unflatten(-1, (G, d))
        w = None if form == "no weight" else _t(1 + 0.2 * r.standard_normal((G, d) if form == "per group" else d), types[1])
        g = _t(r.standard_normal((B, n, G, d)), types[1])
        out = hla.gated_norm_forward(y, z, w, 1e-3, first, types[1])
        assert out.dtype == types[1] and out.is_contiguous()
        grads = hla.gated_norm_backward(y, z, w, g, 1e-3, first)
        _gn_check(y, z, w, 1e-3, first, g, out, grads, form)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", [(1, 70, 2, 8208), (2, 67, 1, 9001)])
def test_gated_norm_of_many_wide_rows(size, types):
    """More rows than the shares of the weight's sums, which a kernel of their own forms."""
    test_gated_norm(size, types, False)
    test_gated_norm(size, types, True)


# ----------------------------------------------------------------------------
RN_SIZES = [(1, 1, 8), (2, 3, 64), (1, 70, 333), (3, 5, 1024), (2, 2, 1001), (1, 9, 2048), (1, 3, 4096), (1, 2, 8192),
            (2, 2, 7777), (1, 2, 16384), (1, 3, 1)]


def _rn_check(x, y, w, post, scale, alpha, eps, go, gr, outs, grads, what):
    xn, yn, wn, pn, sn, gn, rn = map(_n, (x, y, w, post, scale, go, gr))
    one = np.ones(x.shape[-1])
    w1, s1 = (np.abs(one if t is None else t) for t in (wn, sn))
    out, r = O.residual_norm(xn, yn, wn, pn, sn, alpha, eps)
    invy = O.inverse_rms(yn, eps)
    u = np.abs(yn) if pn is None else np.abs(pn * yn * invy)
    size = np.abs(xn) + alpha * s1 * u
    rr = O.inverse_rms(r, eps)
    # 1 / rms(r) is off by the mean of r times r's own error
    rel = 1 + (size * np.abs(r)).mean(-1, keepdims=True) * rr * rr
    hat = size * rr * rel
    _within(outs[0], out, hat * w1, what=what + " out")
    _within(outs[1], r, size, what=what + " r")
    gn, rn = (np.zeros_like(xn) if t is None else t for t in (gn, rn))
    ref = O.residual_norm_vjp(xn, yn, wn, pn, sn, alpha, eps, gn, rn)
    gw = np.abs(gn) * w1
    dr = np.abs(rn) + rr * rel * (gw + hat * (gw * hat).mean(-1, keepdims=True))
    _within(grads[0], ref[0], dr, what=what + " dx")
    du = alpha * s1 * dr
    yh = np.abs(yn) * invy
    dy = du if pn is None else invy * (du * np.abs(pn) + yh * (du * np.abs(pn) * yh).mean(-1, keepdims=True))
    _within(grads[1], ref[1], dy, what=what + " dy")
    for got, r1, terms, there in ((grads[2], ref[2], np.abs(gn) * hat, wn), (grads[3], ref[3], du * yh, pn),
                                  (grads[4], ref[4], alpha * u * dr, sn)):
        assert (got is None) == (there is None)
        if got is not None:
            _within(got, r1, terms.sum((0, 1)), what=what + " weights")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", RN_SIZES)
def test_residual_norm(size, types):
    B, n, D = size
    for form in ("all", "plain", "post", "scale", "strided", "no out", "no r"):
        _say(f"residual norm {size} {types} {form}")
        r = _rng(2, *size)
        x, y, gr, go = (_t(r.standard_normal(size), t) for t in (types[0], types[1], types[0], types[1]))
        if form == "strided":            # views of wider rows, sequences apart
            y = _t(r.standard_normal((B, n + 1, 2 * D)), types[1])[:, 1:, D:]
        w = None if form == "plain" else _t(1 + 0.2 * r.standard_normal(D), types[1])
        post = _t(1 + 0.2 * r.standard_normal(D), types[1]) if form in ("all", "post", "no out", "no r") else None
        scale = _t(0.5 + 0.1 * r.standard_normal(D), types[1]) if form in ("all", "scale", "strided") else None
        alpha = 0.5 if form in ("scale", "strided") else 1.0
        go, gr = None if form == "no out" else go, None if form == "no r" else gr
        outs = hla.residual_norm_forward(x, y, w, post, scale, alpha, 1e-3)
        assert (outs[0].dtype, outs[1].dtype) == (types[1], types[0])
        grads = hla.residual_norm_backward(x, y, w, post, scale, go, gr, alpha, 1e-3)
        _rn_check(x, y, w, post, scale, alpha, 1e-3, go, gr, outs, grads, form)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", [(1, 150, 8208), (2, 70, 9001)])
def test_residual_norm_of_many_wide_rows(size, types):
    test_residual_norm(size, types)


# ----------------------------------------------------------------------------
GLR_SIZES = [(1, 1, 16), (2, 3, 40), (1, 17, 33), (3, 130, 64), (2, 257, 15), (1, 300, 1), (5, 2, 7), (1, 1000, 24),
             (2, 1025, 32), (1, 3001, 18), (1, 5000, 5)]


def _glr_case(B, n, D, dtype, bias, seed):
    r = _rng(seed, B, n, D)
    x, dy = (_t(r.standard_normal((B, n, D)), dtype) for _ in range(2))
    fg = _t(1.5 * r.standard_normal((B, n, 2 * D)), dtype)
    decay = _t(np.log(np.expm1(-np.log(r.uniform(0.9, 0.999, D)) / 8)))
    fb, gb = (_t(0.5 * r.standard_normal(D)) if bias else None for _ in range(2))
    return x, fg[..., :D], fg[..., D:], decay, fb, gb, dy, _t(r.standard_normal((B, D)))


def _glr_size(args, state=None):
    """The recurrence over absolute values."""
    return O.glr(np.abs(args[0]), *args[1:], 8.0, None if state is None else np.abs(state))[0]


def _glr_grad_sizes(args, dy):
    x, f, g, decay, fb, gb = args
    r, i, L, a, root = O.glr_gates(x, f, g, decay, fb, gb, 8.0)
    h = _glr_size(args)
    before = np.concatenate([np.zeros_like(h[:, :1]), h[:, :-1]], 1)
    lam, later = np.empty_like(h), 0
    for t in reversed(range(x.shape[1])):
        lam[:, t] = np.abs(dy[:, t]) + later
        later = a[:, t] * lam[:, t]
    dL = lam * (a * before + i * np.abs(x) * a * a / root)
    df, dg = dL * -L * (1 - r), lam * root * i * np.abs(x) * (1 - i)
    return lam * root * i, df, dg, (dL * 8 * r).sum((0, 1)) * O.sigmoid(decay), df.sum((0, 1)), dg.sum((0, 1))


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", GLR_SIZES)
def test_recurrence(size, dtype, bias):
    B, n, D = size
    _say(f"recurrence {size} {dtype} bias={bias}")
    x, f, g, decay, fb, gb, dy, state = _glr_case(B, n, D, dtype, bias, 3)
    args = [_n(t) for t in (x, f, g, decay, fb, gb)]
    bar = (n + 64) * 2.0 ** -23
    _within(hla.glr_forward(x, f, g, decay, fb, gb), O.glr(*args)[0], _glr_size(args), bar, "from zero")
    sn = _n(state)
    ref, last = O.glr(*args, 8.0, sn)
    size = _glr_size(args, sn)
    _within(hla.glr_prefill(state, x, f, g, decay, fb, gb), ref, size, bar, "from a state")
    _within(state, last, size[:, -1], bar, "state")
    grads = hla.glr_backward(x, f, g, decay, fb, gb, dy)
    names = ("dx", "df", "dg", "ddecay", "df_bias", "dg_bias")
    for name, got, ref, size in zip(names, grads, O.glr_vjp(*args, 8.0, _n(dy)), _glr_grad_sizes(args, _n(dy))):
        if got is not None:
            _within(got, ref, size, 2 * bar, name)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("D", [64, 37, 1])
def test_steps_of_the_recurrence_follow_a_prompt(D, dtype):
    x, f, g, decay, fb, gb, _, state = _glr_case(3, 24, D, dtype, True, 4)
    args = [_n(t) for t in (x, f, g, decay, fb, gb)]
    ref, last = O.glr(*args, 8.0, _n(state))
    size = _glr_size(args, _n(state))
    bar = (24 + 64) * 2.0 ** -23
    got = [hla.glr_prefill(state, x[:, :20], f[:, :20], g[:, :20], decay, fb, gb)]
    for t in range(20, 24):
        got.append(hla.glr_step(state, x[:, t], f[:, t], g[:, t], decay, fb, gb)[:, None])
    _within(torch.cat(got, 1), ref, size, bar)
    _within(state, last, size[:, -1], bar)


# ----------------------------------------------------------------------------
GLU_SIZES = [(1, 1, 8, 8), (2, 3, 64, 40), (1, 17, 72, 136), (4, 1, 256, 512), (1, 64, 136, 72), (1, 65, 1032, 264),
             (3, 100, 200, 1000), (1, 300, 520, 328), (2, 257, 96, 24), (1, 1000, 40, 264), (2, 33, 2048, 16)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("size", GLU_SIZES)
def test_projections(size, act):
    B, n, D, F = size
    _say(f"projections {size} {act}")
    r = _rng(5, *size)
    x, wg, wu = _t(r.standard_normal((B, n, D)), BF16), *(_t(r.standard_normal((F, D)) * D ** -0.5, BF16) for _ in range(2))
    dh = _t(r.standard_normal((B, n, F)), BF16)
    xn, gn, un, dn = map(_n, (x, wg, wu, dh))
    pabs, uabs = np.abs(xn) @ np.abs(gn).T, np.abs(xn) @ np.abs(un).T
    p, u = xn @ gn.T, xn @ un.T
    a, d = O.act(p, act)
    _within(hla.glu_forward(x, wg, wu, act), a * u, 1.13 * pabs * np.abs(u) + np.abs(a) * uabs + np.abs(a * u))
    dx, dwg, dwu, dp, du = O.glu_vjp(xn, gn, un, act, dn)
    # dp and du: their own rounding, and what the sums before them are off by
    ep = 2.0 ** -8 * np.abs(dp) + 2 * FINE * np.abs(dn) * (uabs * np.abs(d) + np.abs(u) * pabs + np.abs(u * d))
    eu = 2.0 ** -8 * np.abs(du) + 2 * FINE * np.abs(dn) * (1.13 * pabs + np.abs(a))
    ep, eu = ep + FINE * np.abs(dp), eu + FINE * np.abs(du)
    rows = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    sizes = (ep @ np.abs(gn) + eu @ np.abs(un), rows(ep).T @ rows(np.abs(xn)), rows(eu).T @ rows(np.abs(xn)))
    for name, got, ref, size in zip(("dx", "dw_gate", "dw_up"), hla.glu_backward(x, wg, wu, dh, act), (dx, dwg, dwu), sizes):
        _within(got, ref, size, 1.0, name)
        if ref.size >= 4096:
            assert np.linalg.norm(_n(got) - ref) <= 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(ref), name


# Every way the work is split, against the products in fp64 on the GPU: tiles of 128, 192 and 256 tokens (the rule
# of the launch, by the CUs that they fill), single steps of k, sums over cut k with a ragged last part.
GLU_SPLITS = [(1, 700, 1088, 328), (1, 2001, 136, 5464), (1, 4100, 64, 4096), (1, 16390, 72, 1032), (1, 5000, 72, 136),
              (1, 1100, 1544, 1096)]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("size", GLU_SPLITS)
def test_projections_in_parts(size, apart):
    B, n, D, F = size
    _say(f"projections {size} apart={apart}")
    gen = torch.Generator("cuda").manual_seed(n)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    if apart:                             # rows of wider rows, sequences with a gap between them
        B, n = 3, -(-n // 3)
        x = draw(B, n + 5, D + 24).to(BF16)[:, 2:-3, 8:-16]
        dh = draw(B, n + 1, F + 8).to(BF16)[:, 1:, 8:]
    else:
        x, dh = draw(B, n, D).to(BF16), draw(B, n, F).to(BF16)
    wg, wu = ((draw(F, D) * D ** -0.5).to(BF16) for _ in range(2))
    xd, gd, ud, dd = (t.double().flatten(0, -2) for t in (x, wg, wu, dh))
    p, u = xd @ gd.T, xd @ ud.T
    s = torch.sigmoid(p)
    dp, du = dd * u * s * (1 + p * (1 - s)), dd * p * s
    refs = (p * s * u, dp @ gd + du @ ud, dp.T @ xd, du.T @ xd)
    got = (hla.glu_forward(x, wg, wu), *hla.glu_backward(x, wg, wu, dh))
    pabs, uabs = xd.abs() @ gd.abs().T, xd.abs() @ ud.abs().T
    ep = (2.0 ** -8 + FINE) * dp.abs() + 2 * FINE * dd.abs() * (uabs * 1.13 + u.abs() * pabs + u.abs() * 1.13)
    eu = (2.0 ** -8 + FINE) * du.abs() + 2 * FINE * dd.abs() * (1.13 * pabs + (p * s).abs())
    sizes = (FINE * (1.13 * pabs * u.abs() + (p * s).abs() * uabs + (p * s * u).abs()), ep @ gd.abs() + eu @ ud.abs(),
             ep.T @ xd.abs(), eu.T @ xd.abs())
    for name, a, r, size in zip(("h", "dx", "dw_gate", "dw_up"), got, refs, sizes):
        a = a.double().reshape(r.shape)
        off = (a - r).abs() - 2.0 ** -8 * (1 + 2.0 ** -7) * r.abs() - size
        assert off.max() <= 0, (name, off.max().item())
        assert (a - r).norm() <= 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * r.norm(), name


# Every way the recurrence is cut, against the oracle: whole and half memory lines a row, sequences in one piece and in
# segments, the last of them short, tiles that end inside a run.
GLR_CUTS = [(1, 4096, 8200), (3, 700, 5472), (1, 4099, 4112), (1, 5003, 200), (1, 9001, 33), (2, 4500, 70), (9, 130, 3650)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", GLR_CUTS)
def test_recurrence_in_parts(size, dtype):
    B, n, D = size
    _say(f"recurrence in parts {size} {dtype}")
    x, f, g, decay, fb, gb, dy, state = _glr_case(B, n, D, dtype, True, 6)
    some = np.unique(np.concatenate([np.arange(min(D, 40)), np.arange(max(0, D - 40), D), np.arange(0, D, max(1, D // 40))]))
    args = [_n(t)[..., some] for t in (x, f, g, decay, fb, gb)]
    bar = (n + 64) * 2.0 ** -23
    sn = _n(state)[:, some]
    ref, last = O.glr(*args, 8.0, sn)
    scale = _glr_size(args, sn)
    got = hla.glr_prefill(state, x, f, g, decay, fb, gb)
    pick = torch.from_numpy(some).cuda()
    _within(got[..., pick], ref, scale, bar, "from a state")
    _within(state[:, pick], last, scale[:, -1], bar, "state")
    grads = hla.glr_backward(x, f, g, decay, fb, gb, dy)
    names = ("dx", "df", "dg", "ddecay", "df_bias", "dg_bias")
    dyn = _n(dy)[..., some]
    for name, a, r, scale in zip(names, grads, O.glr_vjp(*args, 8.0, dyn), _glr_grad_sizes(args, dyn)):
        _within(a[..., pick], r, scale, 2 * bar, name)
