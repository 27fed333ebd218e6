"""Torch-facing helpers for the operators of a block around its mixer: the norm
of the mixer's output with its gate, the residual addition with the norms on
both sides of it, the gated linear recurrence (a mixer of its own), and the
gated feed-forward projections.

torch supplies device memory and the current HIP stream; the computation runs
in libhla.so.  Activations are [B, n, ...] views with any strides between
batches and tokens; outputs are new contiguous tensors.  gated_norm,
residual_norm, glr_scan and glu are differentiable once, in reverse mode:
forward mode, function transforms and second derivatives are refused.
"""
import torch

from . import capi
from .autograd import once
from .mixer import _CODES, _code, _launch, _learns, _on_gpu, _out, _ptr, _rows, _same, _space, _upstream


def _weights_type(*weights):
    """The type of the first weight given; they are held to it."""
    wtype = torch.float32
    for w in weights:
        if w is not None:
            wtype = w.dtype
            break
    if wtype not in _CODES:
        raise TypeError(f"weights must be float32 or bfloat16, got {wtype}")
    return wtype


def _fresh(like, dtype=None):
    """An output of this shape, contiguous (torch.empty takes twice as long)."""
    return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)


# ----------------------------------------------------------------------------
# Norm of a mixer's output with its gate
def _rows3(name, t):
    """(address, elements between batches, tokens, groups) of t [B, n, G, d]."""
    B, n, G, d = t.shape
    bs, ts, gs, one = t.stride()
    if d != 1 and one != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous, got shape {tuple(t.shape)} with strides "
                         f"{t.stride()}")
    return t.data_ptr(), bs if B != 1 else 0, ts if n != 1 else 0, gs if G != 1 else 0


def _gated_args(y, z, weight, dtype):
    """The leading C arguments, the sizes and the codes of a call."""
    if y.dim() != 4:
        raise ValueError(f"y must have 4 dimensions [B, n, groups, d], got shape {tuple(y.shape)}")
    B, n, G, d = y.shape
    _same("z", z, y.shape, dtype, y.device)
    per_group = int(weight is not None and weight.dim() == 2)
    _same("weight", weight, (G, d) if per_group else (d,), None, y.device, contiguous=True)
    wtype = _weights_type(weight)
    _on_gpu(y)
    code, ycode = _CODES.get(dtype), _code("y", y)
    if code is None:
        raise TypeError(f"out_dtype must be float32 or bfloat16, got {dtype}")
    lead = (*_rows3("y", y), *((None, 0, 0, 0) if z is None else _rows3("z", z)), _ptr(weight))
    return lead, (B, n, G, d, per_group), (ycode, code, _CODES[wtype])


def _out_type(y, z, out_dtype):
    return out_dtype if out_dtype is not None else y.dtype if z is None else z.dtype


def gated_norm_forward(y, z=None, weight=None, eps=1e-6, norm_first=False, out_dtype=None):
    """Norm of a mixer's output y [B, n, G, d] over d with its gate z (same
    shape, optional): weight v / sqrt(mean(v^2) + eps) of v = y silu(z), or with
    norm_first that of v = y, times silu(z).  weight [d] or [G, d].  The result
    [B, n, G, d] has z's type (without a gate y's), or out_dtype, which z must
    have; y may be fp32 beside a bf16 z.  Any strides but the last are taken:
    o.transpose(1, 2) of an attention's [B, G, n, d] is fine."""
    dtype = _out_type(y, z, out_dtype)
    lead, sizes, codes = _gated_args(y, z, weight, dtype)
    out = _fresh(y, dtype)
    _launch(capi.hla_gated_norm, y, *lead, out.data_ptr(), *sizes, int(bool(norm_first)), float(eps), *codes)
    return out


def gated_norm_backward(y, z, weight, dout, eps=1e-6, norm_first=False):
    """Gradients (dy, dz, dweight) of gated_norm_forward for dout; None for a z
    or weight not given.  dy is laid out as y where y has no gaps."""
    lead, sizes, codes = _gated_args(y, z, weight, dout.dtype)
    _same("dout", dout, y.shape, None, y.device, contiguous=True)
    dy = torch.empty_like(y)
    if y.shape[-1] != 1 and dy.stride(-1) != 1:
        dy = _fresh(y)
    dz = None if z is None else _fresh(z)
    dw = None if weight is None else torch.empty_like(weight)
    ws, nb = _space(capi.hla_gated_norm_backward_workspace_bytes(*sizes), y.device)
    _launch(capi.hla_gated_norm_backward, y, *lead, dout.data_ptr(), *_rows3("dy", dy), _ptr(dz), _ptr(dw), *sizes,
            int(bool(norm_first)), float(eps), *codes, ws.data_ptr(), nb)
    return dy, dz, dw


class GatedNorm(torch.autograd.Function):
    """gated_norm_forward as a differentiable op."""

    @staticmethod
    def forward(ctx, y, z, weight, eps, norm_first, out_dtype):
        ctx.save_for_backward(y, z, weight)
        ctx.how = eps, norm_first
        return gated_norm_forward(y, z, weight, eps, norm_first, out_dtype)

    @staticmethod
    @once
    def backward(ctx, dout):
        return (*gated_norm_backward(*ctx.saved_tensors, _upstream(dout), *ctx.how), None, None, None)


def gated_norm(y, z=None, weight=None, eps=1e-6, norm_first=False, out_dtype=None):
    """Differentiable gated_norm_forward (in y, z and weight)."""
    if not _learns(y, z, weight):
        return gated_norm_forward(y, z, weight, eps, norm_first, out_dtype)
    return GatedNorm.apply(y, z, weight, eps, norm_first, out_dtype)


# ----------------------------------------------------------------------------
# Residual addition with the norms on both sides
def _residual_args(x, y, weight, post_weight, scale):
    if x.dim() != 3:
        raise ValueError(f"x must have 3 dimensions [B, n, D], got shape {tuple(x.shape)}")
    _same("y", y, x.shape, None, x.device)
    wtype = _weights_type(weight, post_weight, scale)
    device, row = x.device, x.shape[-1:]
    for name, w in (("weight", weight), ("post_weight", post_weight), ("scale", scale)):
        _same(name, w, row, wtype, device, contiguous=True)
    _on_gpu(x)
    codes = _code("x", x), _code("y", y), _CODES[wtype]
    return (*_rows("x", x, 1), *_rows("y", y, 1), _ptr(weight), _ptr(post_weight), _ptr(scale)), tuple(x.shape), codes


def residual_norm_forward(x, y, weight=None, post_weight=None, scale=None, alpha=1.0, eps=1e-6):
    """The residual stream x [B, n, D] after a block's output y, and the norm
    before the next block: r = x + alpha scale u with u = y, or post_weight y /
    sqrt(mean(y^2) + eps) where post_weight is given; returns (weight r /
    sqrt(mean(r^2) + eps) of y's type, r of x's type).  weight, post_weight and
    scale [D] share a type; x may be fp32 beside a bf16 y."""
    lead, sizes, codes = _residual_args(x, y, weight, post_weight, scale)
    out, r = _fresh(y), _fresh(x)
    _launch(capi.hla_residual_norm, x, *lead, out.data_ptr(), r.data_ptr(), *sizes, float(alpha), float(eps), *codes)
    return out, r


def residual_norm_backward(x, y, weight, post_weight, scale, dout, dr, alpha=1.0, eps=1e-6):
    """Gradients (dx, dy, dweight, dpost_weight, dscale) of residual_norm_forward
    for dout (y's type) and dr (x's type), one of which may be None; None for a
    weight not given."""
    lead, sizes, codes = _residual_args(x, y, weight, post_weight, scale)
    _same("dout", dout, x.shape, y.dtype, x.device, contiguous=True)
    _same("dr", dr, x.shape, x.dtype, x.device, contiguous=True)
    dx, dy = _fresh(x), _fresh(y)
    dws = tuple(None if w is None else torch.empty_like(w) for w in (weight, post_weight, scale))
    ws, nb = _space(capi.hla_residual_norm_backward_workspace_bytes(*sizes), x.device)
    _launch(capi.hla_residual_norm_backward, x, *lead, _ptr(dout), _ptr(dr), dx.data_ptr(), dy.data_ptr(),
            *(_ptr(d) for d in dws), *sizes, float(alpha), float(eps), *codes, ws.data_ptr(), nb)
    return dx, dy, *dws


class ResidualNorm(torch.autograd.Function):
    """residual_norm_forward as a differentiable op."""

    @staticmethod
    def forward(ctx, x, y, weight, post_weight, scale, alpha, eps):
        ctx.save_for_backward(x, y, weight, post_weight, scale)
        ctx.how = alpha, eps
        ctx.set_materialize_grads(False)
        return residual_norm_forward(x, y, weight, post_weight, scale, alpha, eps)

    @staticmethod
    @once
    def backward(ctx, dout, dr):
        if dout is None and dr is None:
            return (None,) * 7
        up = (None if d is None else _upstream(d) for d in (dout, dr))
        return (*residual_norm_backward(*ctx.saved_tensors, *up, *ctx.how), None, None)


def residual_norm(x, y, weight=None, post_weight=None, scale=None, alpha=1.0, eps=1e-6):
    """Differentiable residual_norm_forward (in x, y and the weights)."""
    if not _learns(x, y, weight, post_weight, scale):
        return residual_norm_forward(x, y, weight, post_weight, scale, alpha, eps)
    return ResidualNorm.apply(x, y, weight, post_weight, scale, alpha, eps)


# ----------------------------------------------------------------------------
# Gated linear recurrence
def _glr_args(x, f, g, decay, f_bias, g_bias, rank):
    if x.dim() != rank:
        raise ValueError(f"x must have {rank} dimensions, got shape {tuple(x.shape)}")
    shape, dtype, device = x.shape, x.dtype, x.device
    _same("f", f, shape, dtype, device)
    _same("g", g, shape, dtype, device)
    row = shape[-1:]
    for name, t in (("decay", decay), ("f_bias", f_bias), ("g_bias", g_bias)):
        _same(name, t, row, torch.float32, device, contiguous=True)
    _on_gpu(x)
    return (_rows("x", x, 1), _rows("f", f, 1), _rows("g", g, 1)), (decay.data_ptr(), _ptr(f_bias), _ptr(g_bias)), \
        _code("x", x)


def _glr(state, x, f, g, decay, f_bias, g_bias, c, out, workspace, keep=False):
    (rx, rf, rg), params, code = _glr_args(x, f, g, decay, f_bias, g_bias, 3)
    B, n, D = x.shape
    _same("state", state, (B, D), torch.float32, x.device, contiguous=True)
    out = _out(out, x.shape, x)
    kept = torch.empty(capi.hla_glr_kept_bytes(B, n, D) // 4, dtype=torch.float32, device=x.device) if keep else None
    ws, nb = _space(capi.hla_glr_workspace_bytes(B, n, D), x.device, workspace)
    _launch(capi.hla_glr_forward, x, *rx, *rf, *rg, *params, _ptr(state), out.data_ptr(), _ptr(kept), B, n, D,
            float(c), code, ws.data_ptr(), nb)
    return (out, kept) if keep else out


def glr_forward(x, f, g, decay, f_bias=None, g_bias=None, c=8.0, out=None, workspace=None):
    """Gated linear recurrence of every channel of x [B, n, D] from a zero
    state: with r = sigmoid(f + f_bias), i = sigmoid(g + g_bias) and a =
    exp(-c softplus(decay) r), h_t = a_t h_{t-1} + sqrt(1 - a_t^2) i_t x_t.  f
    and g [B, n, D] of x's type; decay, f_bias, g_bias fp32 [D].  Returns every
    h_t, [B, n, D] of x's type."""
    return _glr(None, x, f, g, decay, f_bias, g_bias, c, out, workspace)


def glr_prefill(state, x, f, g, decay, f_bias=None, g_bias=None, c=8.0, out=None, workspace=None):
    """glr_forward from `state` (fp32 [B, D]), which becomes the state after the
    last token."""
    if state is None:
        raise ValueError("glr_prefill needs a state")
    return _glr(state, x, f, g, decay, f_bias, g_bias, c, out, workspace)


def glr_step(state, x_t, f_t, g_t, decay, f_bias=None, g_bias=None, c=8.0, out=None):
    """One token a sequence: x_t, f_t, g_t [B, D] -> [B, D]; `state` updated in place."""
    (rx, rf, rg), params, code = _glr_args(x_t, f_t, g_t, decay, f_bias, g_bias, 2)
    if state is None:
        raise ValueError("glr_step needs a state")
    _same("state", state, x_t.shape, torch.float32, x_t.device, contiguous=True)
    out = _out(out, x_t.shape, x_t)
    _launch(capi.hla_glr_step, x_t, state.data_ptr(), *rx[:2], *rf[:2], *rg[:2], *params, out.data_ptr(), *x_t.shape,
            float(c), code)
    return out


def glr_backward(x, f, g, decay, f_bias, g_bias, dy, c=8.0, kept=None):
    """Gradients (dx, df, dg, ddecay, df_bias, dg_bias) of glr_forward for dy
    [B, n, D]; None for a bias not given.  kept: what a forward of the same
    inputs kept; without it the forward runs again."""
    (rx, rf, rg), params, code = _glr_args(x, f, g, decay, f_bias, g_bias, 3)
    B, n, D = x.shape
    _same("dy", dy, x.shape, x.dtype, x.device)
    ry = _rows("dy", dy, 1)
    if kept is None:
        kept = _glr(None, x, f, g, decay, f_bias, g_bias, c, None, None, keep=True)[1]
    _same("kept", kept, (capi.hla_glr_kept_bytes(B, n, D) // 4,), torch.float32, x.device, contiguous=True)
    dx, df, dg = _fresh(x), _fresh(x), _fresh(x)
    dd, dfb, dgb = (None if t is None else torch.empty_like(t) for t in (decay, f_bias, g_bias))
    ws, nb = _space(capi.hla_glr_backward_workspace_bytes(B, n, D), x.device)
    _launch(capi.hla_glr_backward, x, *rx, *rf, *rg, *params, kept.data_ptr(), *ry, dx.data_ptr(), df.data_ptr(),
            dg.data_ptr(), dd.data_ptr(), _ptr(dfb), _ptr(dgb), B, n, D, float(c), code, ws.data_ptr(), nb)
    return dx, df, dg, dd, dfb, dgb


class GatedLinearRecurrence(torch.autograd.Function):
    """glr_forward as a differentiable op.  The forward keeps the state before
    every 128 tokens."""

    @staticmethod
    def forward(ctx, x, f, g, decay, f_bias, g_bias, c):
        y, kept = _glr(None, x, f, g, decay, f_bias, g_bias, c, None, None, keep=True)
        ctx.save_for_backward(x, f, g, decay, f_bias, g_bias, kept)
        ctx.c = c
        return y

    @staticmethod
    @once
    def backward(ctx, dy):
        *inputs, kept = ctx.saved_tensors
        return (*glr_backward(*inputs, _upstream(dy), ctx.c, kept), None)


def glr_scan(x, f, g, decay, f_bias=None, g_bias=None, c=8.0):
    """Differentiable glr_forward (in x, f, g, decay and the biases)."""
    if not _learns(x, f, g, decay, f_bias, g_bias):
        return glr_forward(x, f, g, decay, f_bias, g_bias, c)
    return GatedLinearRecurrence.apply(x, f, g, decay, f_bias, g_bias, c)


# ----------------------------------------------------------------------------
# Gated feed-forward projections
_ACTS = {"silu": capi.HLA_ACT_SILU, "gelu": capi.HLA_ACT_GELU}


def _glu_args(x, w_gate, w_up, act):
    if x.dim() != 3:
        raise ValueError(f"x must have 3 dimensions [B, n, D], got shape {tuple(x.shape)}")
    B, n, D = x.shape
    if w_gate.dim() != 2 or w_gate.shape[1] != D:
        raise ValueError(f"w_gate must be (F, {D}), got {tuple(w_gate.shape)}")
    _same("w_gate", w_gate, w_gate.shape, x.dtype, x.device, contiguous=True)
    _same("w_up", w_up, w_gate.shape, x.dtype, x.device, contiguous=True)
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}, got {act!r}")
    _on_gpu(x)
    return _rows("x", x, 1), (B, n, D, w_gate.shape[0]), (_ACTS[act], _code("x", x))


def glu_forward(x, w_gate, w_up, act="silu", out=None):
    """Gated feed-forward projections act(x w_gate^T) * (x w_up^T) of x [B, n, D]
    with w_gate, w_up [F, D] -> [B, n, F], in bf16; act "silu" or "gelu" (by the
    error function).  Both products and the gate are one kernel."""
    rows, sizes, codes = _glu_args(x, w_gate, w_up, act)
    out = _out(out, (*sizes[:2], sizes[3]), x)
    _launch(capi.hla_glu_forward, x, *rows, w_gate.data_ptr(), w_up.data_ptr(), out.data_ptr(), *sizes, *codes)
    return out


def glu_backward(x, w_gate, w_up, dh, act="silu"):
    """Gradients (dx, dw_gate, dw_up) of glu_forward for dh [B, n, F]; both projections are formed again."""
    rows, sizes, codes = _glu_args(x, w_gate, w_up, act)
    _same("dh", dh, (*sizes[:2], sizes[3]), x.dtype, x.device)
    dx = _fresh(x)
    dwg, dwu = torch.empty_like(w_gate), torch.empty_like(w_up)
    ws, nb = _space(capi.hla_glu_backward_workspace_bytes(*sizes), x.device)
    _launch(capi.hla_glu_backward, x, *rows, w_gate.data_ptr(), w_up.data_ptr(), *_rows("dh", dh, 1), dx.data_ptr(),
            dwg.data_ptr(), dwu.data_ptr(), *sizes, *codes, ws.data_ptr(), nb)
    return dx, dwg, dwu


class GatedProjections(torch.autograd.Function):
    """glu_forward as a differentiable op."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up, act):
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.act = act
        return glu_forward(x, w_gate, w_up, act)

    @staticmethod
    @once
    def backward(ctx, dh):
        return (*glu_backward(*ctx.saved_tensors, _upstream(dh), ctx.act), None)


def glu(x, w_gate, w_up, act="silu"):
    """Differentiable glu_forward."""
    if not _learns(x, w_gate, w_up):
        return glu_forward(x, w_gate, w_up, act)
    return GatedProjections.apply(x, w_gate, w_up, act)
