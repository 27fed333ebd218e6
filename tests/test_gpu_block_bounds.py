"""Memory around what the operators of a block write, through the C entries:
outputs inside wider buffers, rows of dy with gaps between them, states, and
workspaces of exactly the bytes asked for, filled with NaN.  What lies around
stays as it was, and the results are the binding's bit for bit, so nothing is
read of a workspace that the call did not write."""
import numpy as np
import pytest
import torch

import paper_2510_27258_amd as hla
from paper_2510_27258_amd import capi
from tests.test_gpu_block import BF16, FP32, TYPES, _glr_case, _rng, _say, _t
from tests.test_gpu_block_edges import _same

pytestmark = pytest.mark.gpu

AROUND = 512
CODE = {FP32: capi.HLA_FP32, BF16: capi.HLA_BF16}


class Held:
    """A contiguous tensor of this shape inside a wider buffer of threes."""

    def __init__(self, *shape, dtype=BF16, value=None):
        self.n = int(np.prod(shape))
        self.buf = torch.full((self.n + 2 * AROUND,), 3.0, dtype=dtype, device="cuda")
        self.t = self.buf[AROUND:AROUND + self.n].view(shape)
        if value is not None:
            self.t.copy_(value)
        self.p = self.t.data_ptr()

    def whole(self, what):
        assert (self.buf[:AROUND] == 3).all() and (self.buf[AROUND + self.n:] == 3).all(), what


class Space:
    """A workspace of exactly nb bytes, all ones (NaN in every type), in a buffer that goes on."""

    def __init__(self, nb):
        self.nb = nb
        self.buf = torch.full((nb + AROUND,), 255, dtype=torch.uint8, device="cuda")
        self.buf[nb:] = 90
        self.p = self.buf.data_ptr()

    def whole(self, what):
        assert (self.buf[self.nb:] == 90).all(), what


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _check(what, refs, outs, *others):
    torch.cuda.synchronize()
    for k, (ref, out) in enumerate(zip(refs, outs)):
        out.whole((what, k))
        assert _same(ref, out.t), (what, k)
    for o in others:
        o.whole(what)


# groups that do not divide a workgroup's rows, more groups than rows, odd widths, rows of several waves, and of 1024 threads
GN_SIZES = [(2, 3, 7, 20), (1, 3, 300, 24), (1, 5, 3, 71), (2, 2, 2, 333), (1, 3, 2, 2056), (1, 2, 3, 9001), (1, 2, 1, 16384)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", GN_SIZES)
def test_gated_norm(size, types):
    B, n, G, d = size
    t0, t = types
    codes = CODE[t0], CODE[t], CODE[t]
    for per_group in (0, 1):
        _say(f"bounds of the gated norm {size} {types} per_group={per_group}")
        r = _rng(71, *size)
        y, z, g = _t(r.standard_normal(size), t0), _t(r.standard_normal(size), t), _t(r.standard_normal(size), t)
        w = _t(1 + 0.2 * r.standard_normal((G, d) if per_group else d), t)
        rows = lambda u: (u.data_ptr(), n * G * d, G * d, d)  # noqa: E731
        out = Held(*size, dtype=t)
        capi.hla_gated_norm(*rows(y), *rows(z), w.data_ptr(), out.p, B, n, G, d, per_group, 0, 1e-3, *codes, _stream())
        _check("forward", [hla.gated_norm_forward(y, z, w, 1e-3, False, t)], [out])
        # rows of dy in wider ones: groups, tokens and sequences each with a gap behind them
        gs, ts = d + 3, G * (d + 3) + 5
        bs = n * ts + 7
        wide = torch.full((B * bs + AROUND,), 3.0, dtype=t0, device="cuda")
        dy = wide.as_strided(size, (bs, ts, gs, 1))
        dz, dw = Held(*size, dtype=t), Held(*w.shape, dtype=t)
        ws = Space(capi.hla_gated_norm_backward_workspace_bytes(B, n, G, d, per_group))
        capi.hla_gated_norm_backward(*rows(y), *rows(z), w.data_ptr(), g.data_ptr(), dy.data_ptr(), bs, ts, gs, dz.p, dw.p, B, n, G,
                                     d, per_group, 0, 1e-3, *codes, ws.p, ws.nb, _stream())
        ref = hla.gated_norm_backward(y, z, w, g, 1e-3, False)
        _check("gradients", ref[1:], [dz, dw], ws)
        assert _same(ref[0], dy)
        dy.fill_(3.0)
        assert (wide == 3).all()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("size", [(2, 3, 20), (1, 5, 71), (3, 7, 333), (1, 3, 2056), (1, 67, 9001), (1, 2, 16384)])
def test_residual_norm(size, types):
    B, n, D = size
    t0, t = types
    codes = CODE[t0], CODE[t], CODE[t]
    _say(f"bounds of the residual norm {size} {types}")
    r = _rng(72, *size)
    x, y, gr, go = (_t(r.standard_normal(size), k) for k in (t0, t, t0, t))
    ws3 = [_t(1 + 0.2 * r.standard_normal(D), t) for _ in range(3)]
    rows = lambda u: (u.data_ptr(), n * D, D)  # noqa: E731
    lead = (*rows(x), *rows(y), *(w.data_ptr() for w in ws3))
    outs = [Held(*size, dtype=t), Held(*size, dtype=t0)]
    capi.hla_residual_norm(*lead, *(o.p for o in outs), B, n, D, 0.5, 1e-3, *codes, _stream())
    _check("forward", hla.residual_norm_forward(x, y, *ws3, 0.5, 1e-3), outs)
    outs = [Held(*size, dtype=t0), Held(*size, dtype=t)] + [Held(D, dtype=t) for _ in range(3)]
    ws = Space(capi.hla_residual_norm_backward_workspace_bytes(B, n, D))
    capi.hla_residual_norm_backward(*lead, go.data_ptr(), gr.data_ptr(), *(o.p for o in outs), B, n, D, 0.5, 1e-3, *codes, ws.p,
                                    ws.nb, _stream())
    _check("gradients", hla.residual_norm_backward(x, y, *ws3, go, gr, 0.5, 1e-3), outs, ws)


# one piece and several segments, single channels and pairs, one token
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", [(1, 1, 1), (2, 131, 40), (1, 5, 71), (3, 7, 2056), (1, 3001, 18), (2, 4500, 33)])
def test_recurrence(size, dtype):
    B, n, D = size
    code = CODE[dtype]
    _say(f"bounds of the recurrence {size} {dtype}")
    x, f, g, decay, fb, gb, dy, st = _glr_case(B, n, D, dtype, True, 73)
    f, g = f.contiguous(), g.contiguous()
    rows = lambda u: (u.data_ptr(), n * D, D)  # noqa: E731
    lead = (*rows(x), *rows(f), *rows(g), decay.data_ptr(), fb.data_ptr(), gb.data_ptr())
    state, y = Held(B, D, dtype=FP32, value=st), Held(B, n, D, dtype=dtype)
    kept = Held(capi.hla_glr_kept_bytes(B, n, D) // 4, dtype=FP32)
    ws = Space(capi.hla_glr_workspace_bytes(B, n, D))
    capi.hla_glr_forward(*lead, state.p, y.p, kept.p, B, n, D, 8.0, code, ws.p, ws.nb, _stream())
    ref_state = st.clone()
    ref = hla.glr_prefill(ref_state, x, f, g, decay, fb, gb)
    _check("from a state", [ref, ref_state], [y, state], kept, ws)
    ws = Space(ws.nb)
    capi.hla_glr_forward(*lead, None, y.p, kept.p, B, n, D, 8.0, code, ws.p, ws.nb, _stream())
    _check("from zero", [hla.glr_forward(x, f, g, decay, fb, gb)], [y], kept, ws)
    assert torch.isfinite(kept.t).all() and not kept.t[:D].any()          # the state before the first token
    outs = [Held(B, n, D, dtype=dtype) for _ in range(3)] + [Held(D, dtype=FP32) for _ in range(3)]
    ws = Space(capi.hla_glr_backward_workspace_bytes(B, n, D))
    capi.hla_glr_backward(*lead, kept.p, *rows(dy), *(o.p for o in outs), B, n, D, 8.0, code, ws.p, ws.nb, _stream())
    _check("gradients", hla.glr_backward(x, f, g, decay, fb, gb, dy), outs, ws)
    state, y = Held(B, D, dtype=FP32, value=st), Held(B, D, dtype=dtype)
    capi.hla_glr_step(state.p, x.data_ptr(), n * D, f.data_ptr(), n * D, g.data_ptr(), n * D, *lead[9:], y.p, B, D, 8.0, code,
                      _stream())
    ref_state = st.clone()
    ref = hla.glr_step(ref_state, x[:, 0], f[:, 0], g[:, 0], decay, fb, gb)
    _check("step", [ref, ref_state], [y, state])


# few tokens, tiles, sums in parts, and sequences laid apart, whose tokens the gradients pack
@pytest.mark.parametrize("size", [(1, 3, 72, 40), (2, 300, 40, 328), (1, 700, 1088, 328), (3, 1700, 72, 136)])
def test_projections(size):
    B, n, D, F = size
    _say(f"bounds of the projections {size}")
    r = _rng(74, *size)
    x = _t(r.standard_normal((B, n + 2, D + 8)), BF16)[:, 1:-1, :D]
    wg, wu = (_t(r.standard_normal((F, D)), BF16) for _ in range(2))
    dh = _t(r.standard_normal((B, n, F)), BF16)
    lead = (x.data_ptr(), x.stride(0), x.stride(1), wg.data_ptr(), wu.data_ptr())
    h = Held(B, n, F)
    capi.hla_glu_forward(*lead, h.p, B, n, D, F, capi.HLA_ACT_GELU, capi.HLA_BF16, _stream())
    _check("forward", [hla.glu_forward(x, wg, wu, "gelu")], [h])
    outs = [Held(B, n, D), Held(F, D), Held(F, D)]
    ws = Space(capi.hla_glu_backward_workspace_bytes(B, n, D, F))
    capi.hla_glu_backward(*lead, dh.data_ptr(), n * F, F, *(o.p for o in outs), B, n, D, F, capi.HLA_ACT_GELU, capi.HLA_BF16, ws.p,
                          ws.nb, _stream())
    _check("gradients", hla.glu_backward(x, wg, wu, dh, "gelu"), outs, ws)
