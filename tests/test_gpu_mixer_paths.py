"""Every way the operators around the attention split their work, against the
fp64 oracles: convolution runs of 8 and 16 tokens, several heads a thread of
the norm and rotation, several heads a workgroup of the scan's gradients, many
segments at the widest state.  Bars as in test_gpu_mixer.py.

The scan's gradients at these lengths are compared with the token by token
recurrence in fp64 on the GPU, which is itself held to the oracle."""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from oracle import mixer as O
from tests.test_gpu_mixer import (BF16, FP32, _check_scan, _conv_case, _conv_scale, _n, _qk_case, _qk_scale, _say,
                                  _ssm_case, _within)

pytestmark = pytest.mark.gpu


# B n D K: four channels a thread in runs of 8, and of 16, one channel in runs of 16
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", [(1, 4100, 1024, 4), (2, 4101, 1024, 3), (3, 2201, 333, 2), (3, 2201, 333, 4)])
def test_conv_in_longer_runs(case, dtype):
    B, n, D, K = case
    _say(f"conv {case} {dtype}")
    (x, w, b, _, st), (xn, wn, bn, _, sn) = _conv_case(B, n, D, K, dtype, True, 40)
    bar = 2 ** -8 if dtype == BF16 else 1e-5
    y = hla.conv_prefill(st, x, w, b)
    ref, _, last = O.conv(xn, wn, bn, True, sn)
    _within(y, ref, _conv_scale(xn, wn, bn, True, sn), bar)
    assert np.array_equal(_n(st), last)


# Tokens and heads enough for eight heads a thread forward and four in the
# gradients (2^20 and 2^19 lanes), in heads that are no multiple of either.
MANY = [(2, 2100, 13, 3, 128, 128), (1, 4500, 9, 6, 80, 40), (1, 8300, 5, 3, 64, 32)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", MANY)
def test_qk_several_heads_a_thread(case, dtype, interleaved):
    B, n, H, Hk, d, rot = case
    lanes = 4
    while lanes * (8 if dtype == BF16 else 4) < d:
        lanes *= 2
    assert B * n * (H + Hk) * lanes >= (1 << 19)
    _say(f"qk {case} {dtype} interleaved={interleaved} lanes={B * n * (H + Hk) * lanes / (1 << 20):.2f} * 2^20")
    q, k, qw, kw, cos, sin, pos, gq, gk = _qk_case(*case, dtype, 41)
    outs = hla.qk_norm_rope_forward(q, k, qw, kw, cos, sin, pos, 1e-3, interleaved)
    grads = hla.qk_norm_rope_backward(q, k, qw, kw, cos, sin, pos, gq, gk, 1e-3, interleaved)
    c, s = (_n(t)[pos.cpu().numpy()] for t in (cos, sin))
    bar = 2 ** -8 if dtype == BF16 else 1e-5
    for i, (x, w, g) in enumerate(((q, qw, gq), (k, kw, gk))):
        xn, wn, gn = _n(x), _n(w), _n(g)
        ref = O.norm_rope(xn, wn, c, s, 1e-3, interleaved)
        _within(outs[i], ref, _qk_scale(ref), bar, "out")
        dx, dw = O.norm_rope_vjp(xn, wn, c, s, 1e-3, interleaved, gn)
        inv = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True) + 1e-3)
        size = 2 * inv * (np.abs(gn).max(-1) * np.abs(wn).max()).transpose(0, 2, 1)[..., None]
        size = size * (1 + np.abs(xn * inv).max(-1, keepdims=True))
        _within(grads[i], dx, np.abs(dx) + 1e-3 * size if dtype == BF16 else size, bar, "dx")
        rows = 2 * np.abs(gn).max(-1)[..., None] * np.abs(xn * inv).transpose(0, 2, 1, 3)
        _within(grads[2 + i], dw, np.abs(dw) * (bar if dtype == BF16 else 0) / 1e-5 + rows.sum((0, 1, 2)), 1e-5, "dw")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n", [800, 2100])
def test_widest_scan_over_segments(dtype, n):
    """P = N = 128 in 3 and 8 segments of bf16, 6 and 16 of fp32: each walk
    sums the ends before it, or they are summed once."""
    args, state, _ = _ssm_case(1, n, 2, 128, 128, 1, dtype, 42)
    _check_scan(args, None, hla.ssm_forward(*args), None)
    first = state.clone()
    y = hla.ssm_prefill(state, *args)
    _check_scan(args, first, y, state)


def _vjp64(args, softplus, dy, absolute=False):
    """oracle.mixer.ssm_vjp on the GPU in fp64."""
    x, dt, A, Bm, Cm, D, bias = (a.detach().double() for a in args)
    dy = dy.double()
    if absolute:
        x, Bm, Cm, D, dy = x.abs(), Bm.abs(), Cm.abs(), D.abs(), dy.abs()
    B, n, H, P = x.shape
    G, N = Bm.shape[2:]
    kb, kc = (m.repeat_interleave(H // G, 2) for m in (Bm, Cm))
    raw = dt + bias
    step = torch.logaddexp(raw, torch.zeros_like(raw)) if softplus else raw
    decay = (step * A).exp()
    states = [x.new_zeros(B, H, N, P)]
    for t in range(n):
        states.append(decay[:, t, :, None, None] * states[-1] +
                      kb[:, t, :, :, None] * (step[:, t, :, None] * x[:, t])[:, :, None])
    g = torch.zeros_like(states[0])
    dx, db, dc, dstep, da = (torch.zeros_like(m) for m in (x, kb, kc, step, step))
    for t in reversed(range(n)):
        g = g + kc[:, t, :, :, None] * dy[:, t, :, None]
        dc[:, t] = (states.pop() * dy[:, t, :, None]).sum(-1)
        db[:, t] = step[:, t, :, None] * (g * x[:, t, :, None]).sum(-1)
        du = (g * kb[:, t, :, :, None]).sum(2)
        dx[:, t] = step[:, t, :, None] * du + D[:, None] * dy[:, t]
        g = decay[:, t, :, None, None] * g
        da[:, t] = (g * states[-1]).sum((-1, -2))
        dstep[:, t] = (A.abs() if absolute else A) * da[:, t] + (du * x[:, t]).sum(-1)
    ddt = dstep * (torch.sigmoid(raw) if softplus else 1.0)
    dA = ((step.abs() if absolute else step) * da).sum((0, 1))
    db, dc = (m.reshape(B, n, G, H // G, N).sum(3) for m in (db, dc))
    return [_n(m) for m in (dx, ddt, dA, db, dc, (dy * x).sum((0, 1, 3)), ddt.sum((0, 1)))]


@pytest.mark.parametrize("softplus", [True, False])
def test_the_reference_on_the_gpu_is_the_oracle(softplus):
    args, _, dy = _ssm_case(2, 40, 4, 32, 16, 2, BF16, 43)
    args = list(args)
    if not softplus:
        args[1], args[6] = args[1].abs() * 0.1, args[6] * 0
    for absolute in (False, True):
        want = O.ssm_vjp(*(_n(a) for a in args), softplus, _n(dy), absolute=absolute)
        for a, b in zip(_vjp64(args, softplus, dy, absolute), want):
            assert np.abs(a - b).max() <= 1e-12 * np.abs(b).max()


# B n H P N G, and the heads a workgroup takes (the last of a group's may take fewer)
HEADS = [
    ((1, 540, 64, 16, 16, 1), 3),       # 22 subsets of 3 heads, the last of 1
    ((22, 330, 2, 32, 32, 1), 2),       # no subsets, ragged tiles
    ((3, 1400, 5, 32, 64, 1), 2),       # 3 subsets of 2, 2 and 1; five segments, whose ends are summed once
    ((1, 8250, 4, 64, 128, 2), 2),      # no subsets, groups; 32 segments
    ((7, 1100, 3, 128, 128, 1), 2),     # the widest, in subsets of 2 and 1
    ((1, 8250, 2, 128, 128, 1), 2),     # the widest, no subsets, 32 segments
    ((20, 450, 9, 48, 80, 1), 9),       # odd widths: more heads than waves
]


@pytest.mark.parametrize("case,per", HEADS)
def test_scan_gradients_of_several_heads_a_workgroup(case, per):
    B, n, H, P, N, G = case
    groups, share = B * ((n + 63) // 64) * G, H // G
    subsets = min(share, 1 if groups >= 256 else 256 // groups)
    assert -(-share // subsets) == per      # the kernel's own rule, so that the case is the one named
    _say(f"scan gradients {case}: {per} heads a workgroup")
    args, _, dy = _ssm_case(*case, BF16, 44)
    got = hla.ssm_backward(*args, dy)
    ref, scale = _vjp64(args, True, dy), _vjp64(args, True, dy, absolute=True)
    for name, g, e, s in zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dbias"), got, ref, scale):
        if name in ("dx", "dB", "dC"):
            _within(g, e, s, 2 ** -7, name)
        elif name == "ddt":
            _within(g, e, np.abs(e) + (1e-5 * 2 ** 8) * s, 2 ** -8, name)
        else:
            _within(g, e, s, 1e-5, name)


# No part of dB and dC is rounded before the output but the heads' weighted
# scores, which are held in two pieces (2^-16 of a term); with 1e-5 of the
# terms for the fp32 sums and 2^-8 of the value for the output:
@pytest.mark.parametrize("case", [(2, 130, 4, 64, 64, 1), (1, 300, 2, 128, 128, 1), (1, 200, 6, 16, 48, 2), (22, 330, 2, 32, 32, 1)])
def test_scan_gradients_of_shared_inputs_are_rounded_once(case):
    _say(f"scan gradients {case}")
    args, _, dy = _ssm_case(*case, BF16, 45)
    got = hla.ssm_backward(*args, dy)
    ref, scale = _vjp64(args, True, dy), _vjp64(args, True, dy, absolute=True)
    for i, name in ((3, "dB"), (4, "dC")):
        _within(got[i], ref[i], 2 ** -8 * np.abs(ref[i]) + 3e-5 * scale[i], 1, name)


@pytest.mark.parametrize("P,N", [(32, 32), (64, 128), (128, 128)])
def test_steps_before_all_pairs_have_no_gradient(P, N):
    """x at the tokens 61 and 62 of a tile and dy at 62 and 63: the decay of a
    token up to 61 lies between no pair, and its step has no gradient.  What a
    kernel adds and takes away again there has to cancel to fp64's 2^-53 of at
    most 64 x 64 terms, 5e-13 of the largest gradient."""
    x, dt, A, Bm, Cm, D, bias = _ssm_case(1, 64, 3, P, N, 1, BF16, 46, dt_dtype=FP32, views=False)[0]
    x[:, :61], x[:, 63:] = 0, 0
    dy = torch.zeros_like(x)
    dy[:, 62:] = torch.randn(dy[:, 62:].shape, device="cuda").to(BF16)
    ddt = hla.ssm_backward(x, dt, A, Bm, Cm, D, bias, dy)[1]
    assert (ddt[:, :61].abs().amax((0, 1)) <= 1e-12 * ddt.abs().amax((0, 1))).all(), ddt[0, :, 0]


def test_keys_past_32_bits():
    """Keys of more than 2^32 bytes and 2^31 elements, of 61 heads (no multiple
    of what a thread takes): the last rows against the same rows by themselves."""
    n, Hk = 280000, 61
    k = torch.empty(1, n, Hk, 128, dtype=BF16, device="cuda")
    k.normal_(generator=torch.Generator("cuda").manual_seed(1))
    ang = torch.arange(1000, device="cuda")[:, None] * 100.0 ** (-torch.arange(64, device="cuda") / 64)
    pos = torch.arange(n, device="cuda")[None] % 1000
    args = None, None, ang.cos(), ang.sin()
    qo, ko = hla.qk_norm_rope_forward(k[:, :, :1], k, *args, pos)
    qt, kt = hla.qk_norm_rope_forward(k[:, -100:, :1], k[:, -100:], *args, pos[:, -100:])
    assert torch.equal(ko[:, :, -100:], kt) and torch.equal(qo[:, :, -100:], qt)
