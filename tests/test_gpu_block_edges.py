"""Extreme values, addresses, strides, lengths beyond 32-bit offsets, streams
and captured graphs through the operators of a block.  Bars as in
test_gpu_block.py, where values are compared with the oracles; elsewhere the
same call on the same values has to give the same bits, since every sum has a
fixed order."""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from oracle import block as O
from paper_2510_27258_amd import capi
from tests.test_gpu_block import BF16, FP32, _glr_case, _n, _rng, _say, _t, _within

pytestmark = pytest.mark.gpu


def _same(a, b):
    """The same bits, whatever they are (NaN too)."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def _all(outs):
    return [o for o in (outs if isinstance(outs, (tuple, list)) else (outs,)) if o is not None]


def _calls(seed, B=2, n=37, D=72, dtype=BF16):
    """name: (call of its tensors -> outputs, the tensors).  States are copied by the call."""
    r = _rng(seed, B, n, D)
    a = lambda *s, t=dtype: _t(r.standard_normal(s), t)  # noqa: E731
    x, f, g, decay, fb, gb, dy, st = _glr_case(B, n, D, dtype, True, seed)

    def prefill(st, *args):
        st = st.clone()
        return hla.glr_prefill(st, *args), st

    def step(st, x, f, g, *args):
        st = st.clone()
        return hla.glr_step(st, x[:, 0], f[:, 0], g[:, 0], *args), st
    calls = {
        "gated norm": (hla.gated_norm_forward, [a(B, n, 3, D), a(B, n, 3, D), a(D)]),
        "gated norm back": (hla.gated_norm_backward, [a(B, n, 3, D), a(B, n, 3, D), a(3, D), a(B, n, 3, D)]),
        "residual norm": (hla.residual_norm_forward, [a(B, n, D) for _ in range(2)] + [a(D) for _ in range(3)]),
        "residual norm back": (hla.residual_norm_backward, [a(B, n, D) for _ in range(2)] + [a(D) for _ in range(3)] +
                               [a(B, n, D) for _ in range(2)]),
        "recurrence": (prefill, [st, x, f, g, decay, fb, gb]),
        "step": (step, [st, x, f, g, decay, fb, gb]),
        "recurrence back": (hla.glr_backward, [x, f, g, decay, fb, gb, dy]),
    }
    if dtype == BF16 and D % 8 == 0:
        calls["projections"] = (hla.glu_forward, [a(B, n, D), a(88, D), a(88, D)])
        calls["few projections"] = (hla.glu_forward, [a(B, 3, D), a(88, D), a(88, D)])
        calls["projections back"] = (hla.glu_backward, [a(B, n, D), a(88, D), a(88, D), a(B, n, 88)])
    return calls


# of the calls above: named without making one, which takes a GPU
NAMES = ["few projections", "gated norm", "gated norm back", "projections", "projections back", "recurrence", "recurrence back",
         "residual norm", "residual norm back", "step"]


def test_every_call_is_named():
    assert sorted(_calls(0)) == NAMES


# ----------------------------------------------------------------------------
@pytest.mark.parametrize("D", [72, 71])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_any_address_of_the_elements_type(dtype, D):
    """Tensors one element off a 16-byte boundary, also in rows of odd length: what aligned ones give.  The norms keep
    their bits; the recurrence takes single channels instead of pairs, whose runs join at other tokens."""
    for name in ("gated norm", "gated norm back", "residual norm", "residual norm back", "recurrence", "step", "recurrence back"):
        call, args = _calls(11, D=D, dtype=dtype)[name]
        off = []
        for t in args:
            wide = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
            wide[1:] = t.flatten()
            off.append(wide[1:].view(t.shape))
        _say(f"address {name} D={D} {dtype}")
        for u, v in zip(_all(call(*args)), _all(call(*off))):
            if "norm" in name:
                assert _same(u, v)
            else:
                assert torch.allclose(u.float(), v.float(), rtol=2 ** -7 if u.dtype == BF16 else 1e-5, atol=1e-4)


@pytest.mark.parametrize("name", NAMES)
def test_repeated_and_padded_rows(name):
    """Batches, tokens or groups with a stride of zero, and rows of a wider tensor, give what a copy gives."""
    call, args = _calls(12)[name]
    copies = []
    for k, t in enumerate(args):
        if t.dim() < 3 or t.dtype == FP32:
            copies.append([t, t, t])
            continue
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 16), float("nan"), dtype=t.dtype, device="cuda")
        wide[..., 8:-8] = t
        upstream = "back" in name and k == len(args) - 1 or "residual norm back" in name and k >= 5
        copies.append([t[:1].expand(t.shape) if not upstream else t[:1].expand(t.shape).contiguous(),
                       t[:, :1].expand(t.shape) if not upstream else t[:, :1].expand(t.shape).contiguous(),
                       wide[..., 8:-8] if not upstream or "projections" in name or "recurrence" in name else t])
    for k in range(3):
        views = [c[k] for c in copies]
        _say(f"views {name} {k}")
        for u, v in zip(_all(call(*views)), _all(call(*(v.contiguous() for v in views)))):
            assert _same(u, v)


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_rows_that_overlap_keep_bad_values_in_their_channel(which):
    """x, f, g or dy in rows of 64 that begin 32 elements apart: what lies where a token behind the last would is the
    last token's channels 32 to 63.  A NaN there spoils its own channel's sums and no other's."""
    x, f, g, decay, fb, gb, dy, _ = _glr_case(1, 37, 64, FP32, True, 15)
    inputs = [t.contiguous() for t in (x, f, g, dy)]
    flat = torch.randn(36 * 32 + 64, generator=torch.Generator().manual_seed(16)).cuda()
    got = []
    for bad in (False, True):
        if bad:
            flat[36 * 32 + 32 + 3] = float("nan")                       # token 36's channel 35; token 37's channel 3
        inputs[which] = flat.as_strided((1, 37, 64), (0, 32, 1))
        got.append(hla.glr_backward(*inputs[:3], decay, fb, gb, inputs[3]))
    others = torch.arange(64, device="cuda") != 35
    for a, b in zip(*got):
        assert torch.isfinite(b[..., others]).all() and _same(a[..., others], b[..., others])
    assert not torch.isfinite(got[1][3][35])


# ----------------------------------------------------------------------------
def test_zero_rows_and_eps():
    z = torch.zeros(2, 5, 3, 40, device="cuda", dtype=BF16)
    one = torch.ones_like(z)
    assert not hla.gated_norm_forward(z, one).any() and not hla.gated_norm_forward(one, z).any()
    dy, dz, _ = hla.gated_norm_backward(z, one, None, one)
    assert torch.isfinite(dy.float()).all() and torch.isfinite(dz.float()).all()
    assert hla.gated_norm_forward(z, eps=0.0).isnan().all()           # 0 / 0, as the formula says
    x = z[:, :, 0].contiguous()
    out, r = hla.residual_norm_forward(x, x, post_weight=torch.ones(40, device="cuda"))
    assert not out.any() and not r.any()
    grads = hla.residual_norm_backward(x, x, None, torch.ones(40, device="cuda"), None, one[:, :, 0].contiguous(), None)
    assert all(torch.isfinite(g.float()).all() for g in grads if g is not None)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_bad_values_stay_in_their_rows(bad, dtype):
    """One bad element of token 5 of sequence 0: norms and projections lose that token's row (its gradients too), the
    recurrence that channel from the token on; everything else keeps its bits."""
    for name, (call, args) in _calls(13, dtype=dtype).items():
        if name in ("step", "few projections"):
            continue
        which = 1 if name == "recurrence" else 0
        spoilt = [t.clone() if k == which else t for k, t in enumerate(args)]
        spoilt[which].view(2, 37, -1)[0, 5, 3] = bad
        _say(f"bad value {bad} {name} {dtype}")
        clean, got = _all(call(*args)), _all(call(*spoilt))
        for u, v in zip(clean, got):
            if u.dim() < 3:
                if name == "recurrence":                                # the state
                    keep = torch.ones_like(u, dtype=torch.bool)
                    keep[0, 3] = False
                    assert torch.equal(u[keep], v[keep]) and not torch.isfinite(v[0, 3])
                continue                                                # sums over all tokens
            u, v = (t.reshape(2, 37, -1) for t in (u, v))
            keep = torch.ones_like(u, dtype=torch.bool)
            if name == "recurrence":
                keep[0, 5:, 3] = False
                assert not torch.isfinite(v[0, 5:, 3].float()).any()
            elif name == "recurrence back":
                keep[0, :, 3] = False
            else:
                keep[0, 5] = False
            assert torch.equal(u[keep], v[keep])
        if name == "residual norm":
            assert not torch.isfinite(got[1][0, 5, 3].float()) and torch.isfinite(got[1].float()).sum() == got[1].numel() - 1


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gates_and_decays_at_their_ends(dtype):
    """Gates that are shut or wide open, decays that forget nothing or all, c = 0: the limits of the formulas, and
    finite gradients throughout."""
    n, D = 300, 12
    x, f, g, decay, fb, gb, dy, state = _glr_case(2, n, D, dtype, True, 14)
    f = f.contiguous()
    f[..., 0:2], f[..., 2:4] = -float("inf"), 200.0            # keep all; open
    g = g.contiguous()
    g[..., 1], g[..., 3] = -200.0, 200.0
    f[..., 4:6] = -90.0
    decay[5], decay[6], decay[7], decay[8] = -120.0, 60.0, -30.0, 5.0
    args = [_n(t) for t in (x, f, g, decay, fb, gb)]
    for c in (8.0, 0.0):
        st = state.clone()
        y = hla.glr_prefill(st, x, f, g, decay, fb, gb, c)
        ref, last = O.glr(*args, c, _n(state))
        size = O.glr(np.abs(args[0]), *args[1:], c, np.abs(_n(state)))[0]
        bar = (n + 64) * 2.0 ** -23
        _within(y, ref, size, bar)
        _within(st, last, size[:, -1], bar)
        if c == 0.0:
            assert torch.equal(st, state)
        for got in hla.glr_backward(x, f, g, decay, fb, gb, dy, c):
            assert torch.isfinite(got.float()).all()


def test_activations_far_out():
    """Projections whose pre-activations reach +-60: both activations and their derivatives at their limits."""
    D, F = 16, 24
    x = torch.zeros(1, 40, D, device="cuda", dtype=BF16)
    x[0, :, 0] = torch.linspace(-60, 60, 40)
    wg, wu = torch.zeros(F, D, device="cuda", dtype=BF16), torch.zeros(F, D, device="cuda", dtype=BF16)
    wg[:, 0], wu[:, 1] = 1.0, 1.0
    x[0, :, 1] = 1.0
    dh = torch.ones(1, 40, F, device="cuda", dtype=BF16)
    xn, gn, un, dn = map(_n, (x, wg, wu, dh))
    for act in ("silu", "gelu"):
        ref = O.glu(xn, gn, un, act)
        _within(hla.glu_forward(x, wg, wu, act), ref, np.maximum(np.abs(ref), 1e-2), what=act)
        dx, dwg, dwu, _, _ = O.glu_vjp(xn, gn, un, act, dn)
        got = hla.glu_backward(x, wg, wu, dh, act)
        for u, v in zip(got, (dx, dwg, dwu)):
            assert torch.isfinite(u.float()).all()
        # dwu's terms are act(p) x and dwg's act'(p) u x: rounded once each, summed over 40 tokens
        size = np.abs(O.act(xn[..., :1], act)[0]).sum()
        _within(got[2][:, 1], dwu[:, 1], np.full(F, size), 2.0 ** -8 + 1e-5, act)


# ----------------------------------------------------------------------------
def test_nothing_is_written_around_the_outputs():
    """Odd sizes through the C entries, outputs inside wider buffers: the bytes before and behind stay as they were."""
    s = torch.cuda.current_stream().cuda_stream

    def guarded(*shape, dtype=BF16):
        n = int(np.prod(shape))
        buf = torch.full((n + 512,), 3.0, dtype=dtype, device="cuda")
        return buf, buf.data_ptr() + 256 * buf.element_size(), n

    def check(*bufs):
        torch.cuda.synchronize()
        for buf, _, n in bufs:
            assert (buf[:256] == 3).all() and (buf[256 + n:] == 3).all()
            assert not (buf[256:256 + n] == 3).all()
    for B, n, D in ((1, 3, 71), (2, 131, 40), (1, 5, 1), (3, 7, 2056)):
        calls = _calls(15, B, n, D)
        x, f, g, decay, fb, gb, dy, st = _glr_case(B, n, D, BF16, True, 15)
        f, g = f.contiguous(), g.contiguous()
        ws = torch.empty(max(capi.hla_glr_workspace_bytes(B, n, D), capi.hla_glr_backward_workspace_bytes(B, n, D),
                             capi.hla_residual_norm_backward_workspace_bytes(B, n, D)), dtype=torch.uint8, device="cuda")
        kb = capi.hla_glr_kept_bytes(B, n, D) // 4
        y, kept = guarded(B, n, D), guarded(kb, dtype=FP32)
        rows = lambda t: (t.data_ptr(), n * D, D)  # noqa: E731
        capi.hla_glr_forward(*rows(x), *rows(f), *rows(g), decay.data_ptr(), fb.data_ptr(), gb.data_ptr(), None, y[1], kept[1], B, n, D,
                             8.0, 1, ws.data_ptr(), ws.numel(), s)
        check(y, kept)
        outs = [guarded(B, n, D) for _ in range(3)] + [guarded(D, dtype=FP32) for _ in range(3)]
        capi.hla_glr_backward(*rows(x), *rows(f), *rows(g), decay.data_ptr(), fb.data_ptr(), gb.data_ptr(), kept[1], *rows(dy),
                              *(o[1] for o in outs), B, n, D, 8.0, 1, ws.data_ptr(), ws.numel(), s)
        check(*outs)
        a = calls["residual norm back"][1]
        outs = [guarded(B, n, D) for _ in range(2)]
        capi.hla_residual_norm(*rows(a[0]), *rows(a[1]), *(t.data_ptr() for t in a[2:5]), outs[0][1], outs[1][1], B, n, D, 1.0, 1e-6, 1, 1, 1, s)
        check(*outs)
        outs = [guarded(B, n, D) for _ in range(2)] + [guarded(D) for _ in range(3)]
        capi.hla_residual_norm_backward(*rows(a[0]), *rows(a[1]), *(t.data_ptr() for t in a[2:7]), *(o[1] for o in outs), B, n, D, 1.0,
                                        1e-6, 1, 1, 1, ws.data_ptr(), ws.numel(), s)
        check(*outs)
    for B, n, D, F in ((1, 3, 72, 40), (1, 130, 64, 72), (2, 300, 40, 328)):
        r = _rng(16, n)
        x, wg, wu, dh = (_t(r.standard_normal(s_), BF16) for s_ in ((B, n, D), (F, D), (F, D), (B, n, F)))
        ws = torch.empty(capi.hla_glu_backward_workspace_bytes(B, n, D, F), dtype=torch.uint8, device="cuda")
        h = guarded(B, n, F)
        capi.hla_glu_forward(x.data_ptr(), n * D, D, wg.data_ptr(), wu.data_ptr(), h[1], B, n, D, F, 0, 1, s)
        check(h)
        outs = [guarded(B, n, D), guarded(F, D), guarded(F, D)]
        capi.hla_glu_backward(x.data_ptr(), n * D, D, wg.data_ptr(), wu.data_ptr(), dh.data_ptr(), n * F, F, *(o[1] for o in outs), B, n, D,
                              F, 0, 1, ws.data_ptr(), ws.numel(), s)
        check(*outs)


# ----------------------------------------------------------------------------
def test_offsets_past_32_bits():
    """More than 2^32 bytes of every input and output: the last tokens are those of a short call."""
    _say("residual norm")
    w = torch.randn(8192, device="cuda").to(BF16)
    y = torch.zeros(1, 1 << 19, 8192, dtype=BF16, device="cuda")        # 8.6 GB
    y[:, -2:] = torch.randn(2, 8192, device="cuda")
    y[:, :2] = torch.randn(2, 8192, device="cuda")
    out, r = hla.residual_norm_forward(y, y, w)
    short = hla.residual_norm_forward(y[:, -2:].contiguous(), y[:, -2:].contiguous(), w)
    assert _same(out[:, -2:], short[0]) and _same(r[:, -2:], short[1])
    del out, r
    _say("gated norm")
    heads = y.view(1, 1 << 19, 64, 128)
    out = hla.gated_norm_forward(heads, heads, w[:128].contiguous())
    assert _same(out[:, -2:], hla.gated_norm_forward(heads[:, -2:].contiguous(), heads[:, -2:].contiguous(), w[:128].contiguous()))
    dy, dz, dw = hla.gated_norm_backward(heads, heads, w[:128].contiguous(), out)
    short = hla.gated_norm_backward(heads[:, -2:].contiguous(), heads[:, -2:].contiguous(), w[:128].contiguous(), out[:, -2:].contiguous())
    assert _same(dy[:, -2:], short[0]) and _same(dz[:, -2:], short[1])
    del out, dy, dz, heads
    _say("recurrence")
    gate = torch.zeros(1, 1, 8192, dtype=BF16, device="cuda").expand_as(y)
    decay = torch.full((8192,), -2.0, device="cuda")
    state = torch.zeros(1, 8192, device="cuda")
    got = hla.glr_prefill(state, y, gate, gate, decay)
    # the middle is zeros: after 2^19 tokens nothing of the first two is left
    st = torch.zeros(1, 8192, device="cuda")
    ref = hla.glr_prefill(st, y[:, -40:].contiguous(), gate[:, -40:].contiguous(), gate[:, -40:].contiguous(), decay)
    assert torch.allclose(got[:, -2:].float(), ref[:, -2:].float(), rtol=2 ** -7, atol=1e-6)
    assert torch.allclose(state, st, rtol=1e-5, atol=1e-7)
    del got
    grads = hla.glr_backward(y, gate, gate, decay, None, None, y)
    short = hla.glr_backward(*(t[:, -40:].contiguous() for t in (y, gate, gate)), decay, None, None, y[:, -40:].contiguous())
    for a, b in zip(grads[:3], short[:3]):
        assert torch.allclose(a[:, -2:].float(), b[:, -2:].float(), rtol=2 ** -6, atol=1e-5)
    del grads, short, y, gate
    torch.cuda.empty_cache()
    _say("projections")
    m, F = 1 << 18, 8264                                                # 4.3 GB of h, 8.7 of the gradients between
    x = torch.randn(1, m, 64, device="cuda").to(BF16)
    wg, wu = (torch.randn(F, 64, device="cuda").mul_(0.125).to(BF16) for _ in range(2))
    h = hla.glu_forward(x, wg, wu)
    assert _same(h[:, -300:], hla.glu_forward(x[:, -300:].contiguous(), wg, wu))
    dx, dwg, dwu = hla.glu_backward(x, wg, wu, h)
    short = hla.glu_backward(x[:, -300:].contiguous(), wg, wu, h[:, -300:].contiguous())
    assert torch.allclose(dx[:, -300:].float(), short[0].float(), rtol=2 ** -6, atol=2 ** -8)
    assert torch.isfinite(dwg.float()).all() and torch.isfinite(dwu.float()).all()


# ----------------------------------------------------------------------------
@pytest.mark.parametrize("name", NAMES)
def test_other_streams_and_repeats(name):
    """Two calls at once on streams of their own, and again: one result."""
    first, second = _calls(17, n=900), _calls(18, n=900)
    refs = [_all(c[name][0](*c[name][1])) for c in (first, second)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        outs = []
        for s, c in zip(streams, (first, second)):
            with torch.cuda.stream(s):
                outs.append(_all(c[name][0](*c[name][1])))
        torch.cuda.synchronize()
        for got, ref in zip(outs, refs):
            assert all(_same(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("name", NAMES)
def test_captured_graphs(name):
    """Captured once, replayed on new inputs between eager work: the eager results."""
    call, args = _calls(19, n=260)[name]
    args = [t.contiguous() for t in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all(call(*args))
    for k in range(4):
        for t, new in zip(args, _calls(20 + k, n=260)[name][1]):
            t.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        got = [o.clone() for o in outs]
        ref = _all(call(*args))
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(got, ref)), (name, k)


def test_a_captured_training_step():
    """Forward and gradients through autograd in one graph, two graphs in turn."""
    def step(x, p):
        u, f, g = (x * p["in"]).split(64, -1)
        h = hla.glr_scan(u, f, g, p["decay"], p["bias"], p["bias"])
        h = hla.gated_norm(h.unflatten(-1, (4, 16)), u.unflatten(-1, (4, 16)), p["norm"]).flatten(2)
        out, r = hla.residual_norm(u.float(), hla.glu(h, p["gate"], p["up"]), p["w"], p["post"], p["scale"])
        return torch.autograd.grad((out.float() * r).sum(), list(p.values()))

    r = _rng(30)
    p = {"in": _t(r.standard_normal(192), BF16), "decay": _t(r.standard_normal(64) - 3), "bias": _t(r.standard_normal(64)),
         "norm": _t(r.standard_normal((4, 16)), BF16), "gate": _t(r.standard_normal((64, 64)) / 8, BF16),
         "up": _t(r.standard_normal((64, 64)) / 8, BF16), "w": _t(r.standard_normal(64), BF16), "post": _t(r.standard_normal(64), BF16),
         "scale": _t(r.standard_normal(64), BF16)}
    p = {k: v.requires_grad_() for k, v in p.items()}
    graphs = []
    for n in (150, 40):
        x = _t(r.standard_normal((2, n, 192)), BF16)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(x, p)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step(x, p)
        graphs.append((graph, x, outs))
    for k in range(3):
        for graph, x, outs in graphs:
            x.copy_(_t(_rng(40 + k).standard_normal(tuple(x.shape)), BF16))
            graph.replay()
            got = [o.clone() for o in outs]
            ref = step(x, p)
            torch.cuda.synchronize()
            for name, a, b in zip(p, got, ref):
                assert _same(a, b) or torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=1e-6), (name, k)


def _differences(op, args, ups, grads):
    """fp32 directional derivatives by central differences of step 1e-3: off by about its square and 2^-24 over it,
    both below 1e-3 of the terms' absolute sum."""
    r = _rng(51, len(args))
    for k, grad in enumerate(grads):
        d = _t(r.standard_normal(tuple(args[k].shape)))
        vals = []
        for sign in (1, -1):
            outs = _all(op(*(a + sign * 1e-3 * d if j == k else a for j, a in enumerate(args))))
            vals.append(sum((o.double() * u.double()).sum() for o, u in zip(outs, ups)))
        terms = grad.double() * d.double()
        assert ((vals[0] - vals[1]) / 2e-3 - terms.sum()).abs() <= 1e-3 * terms.abs().sum(), k


@pytest.mark.parametrize("first", [False, True])
def test_gated_norm_against_differences(first):
    r = _rng(50)
    y, z, w, g = (_t(r.standard_normal(s)) for s in ((2, 9, 3, 24), (2, 9, 3, 24), (24,), (2, 9, 3, 24)))
    _differences(lambda *a: hla.gated_norm_forward(*a, 1e-3, first), (y, z, w), (g,), hla.gated_norm_backward(y, z, w, g, 1e-3, first))


@pytest.mark.parametrize("alpha", [1.0, 0.5])
def test_residual_norm_against_differences(alpha):
    r = _rng(52)
    x, y, go, gr = (_t(r.standard_normal((2, 9, 40))) for _ in range(4))
    w, p, s = (_t(r.standard_normal(40)) for _ in range(3))
    _differences(lambda *a: hla.residual_norm_forward(*a, alpha, 1e-3), (x, y, w, p, s), (go, gr),
                 hla.residual_norm_backward(x, y, w, p, s, go, gr, alpha, 1e-3))


def test_recurrence_against_differences():
    x, f, g, decay, fb, gb, dy, _ = _glr_case(2, 30, 6, FP32, True, 53)
    args = (x, f.contiguous(), g.contiguous(), decay, fb, gb)
    _differences(hla.glr_forward, args, (dy,), hla.glr_backward(*args, dy))
