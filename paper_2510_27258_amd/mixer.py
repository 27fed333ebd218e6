"""Torch-facing helpers for the operators around the attention: the short
causal convolution, the norm and rotation of queries and keys, and the
selective state space scan.

torch supplies device memory and the current HIP stream; the computation runs
in libhla.so.  Activations are [B, n, ...] views with any strides between
batches and tokens, such as slices of a projection's output; outputs are new
contiguous tensors.  short_conv, qk_norm_rope and ssm_scan are differentiable
once, in reverse mode: forward mode, function transforms and second derivatives
are refused.
"""
import torch
import torch.autograd.forward_ad as _forward_ad

from . import capi
from .autograd import once

_CODES = {torch.float32: capi.HLA_FP32, torch.bfloat16: capi.HLA_BF16}


def _code(name, t):
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return code


def _rows(name, t, inner):
    """(address, elements between batches, elements between tokens) of t, whose
    last `inner` dimensions must be one contiguous row.  The stride of a
    dimension of size one is not used."""
    want = 1
    for i in range(1, inner + 1):
        if t.shape[-i] != 1 and t.stride(-i) != want:
            raise ValueError(f"{name}: the last {inner} dimension(s) must be contiguous, got shape {tuple(t.shape)} "
                             f"with strides {t.stride()}")
        want *= t.shape[-i]
    lead = t.dim() - inner
    bs = t.stride(0) if t.shape[0] != 1 else 0
    ts = t.stride(1) if lead == 2 and t.shape[1] != 1 else 0
    return t.data_ptr(), bs, ts


def _ptr(t):
    return None if t is None else t.data_ptr()


def _same(what, t, shape, dtype=None, device=None, contiguous=False):
    """t, optional, must have this shape (and type, device, layout)."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {tuple(shape)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{what} must be on {device}, got {t.device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")


def _on_gpu(t):
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")


# the device and stream of the calling thread, without torch.cuda's wrappers, which cost a
# decode call more than its kernel
_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(entry, t, *args):
    """entry(*args, the current stream of t's device), with that device current:
    a launch goes to the current device's context."""
    index = t.device.index
    now = _device()
    if now == index:
        entry(*args, _raw_stream(index))
        return
    torch.cuda.set_device(index)
    try:
        entry(*args, _raw_stream(index))
    finally:
        torch.cuda.set_device(now)


def _has_graph(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _learns(*tensors):
    """Whether a call has to go through its autograd function: an input has a
    graph, or may have a tangent (inside a forward-mode level), which that
    function refuses."""
    return getattr(_forward_ad, "_current_level", 0) >= 0 or _has_graph(*tensors)


def _out(out, shape, like, name="out"):
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    _same(name, out, shape, like.dtype, like.device, contiguous=True)
    return out


def _space(nbytes, device, workspace=None):
    """A workspace of nbytes; none for sizes that the query refuses (0), which
    the entry refuses with its own code before it looks at the workspace."""
    if workspace is None or nbytes == 0:
        return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace, workspace.numel() * workspace.element_size()


def _upstream(g):
    """An upstream gradient as the kernels read it: contiguous and on a 16-byte
    boundary, which autograd's views (slices of the gradient of a torch.cat)
    need not be."""
    return g.contiguous() if g.data_ptr() % 16 == 0 else g.clone(memory_format=torch.contiguous_format)


# ----------------------------------------------------------------------------
# Short causal convolution
def _conv_args(x, weight, bias, rank):
    if x.dim() != rank:
        raise ValueError(f"x must have {rank} dimensions, got shape {tuple(x.shape)}")
    D = x.shape[-1]
    if weight.dim() != 2 or weight.shape[0] != D:
        raise ValueError(f"weight must be ({D}, K), got {tuple(weight.shape)}")
    _same("weight", weight, weight.shape, None, x.device, contiguous=True)
    _same("bias", bias, (D,), weight.dtype, x.device, contiguous=True)
    _on_gpu(x)
    return D, weight.shape[1], _code("x", x), _code("weight", weight)


def _conv(x, weight, bias, silu, state, out, rank):
    D, K, code, wcode = _conv_args(x, weight, bias, rank)
    B, n = x.shape[0], x.shape[1] if rank == 3 else 1
    _same("state", state, (B, K - 1, D), x.dtype, x.device, contiguous=True)
    rows = _rows("x", x, 1)
    out = _out(out, x.shape, x)
    _launch(capi.hla_conv_forward, x, *rows, weight.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(), B, n, D,
            K, int(bool(silu)), code, wcode)
    return out


def conv_forward(x, weight, bias=None, silu=True, out=None):
    """Causal convolution of x [B, n, D] with weight [D, K], K = 2 .. 4, from
    zeros: y[b,t,c] = act(bias[c] + sum_j weight[c,j] x[b,t-K+1+j,c]), act
    SiLU or the identity.  y has x's type."""
    return _conv(x, weight, bias, silu, None, out, 3)


def conv_prefill(state, x, weight, bias=None, silu=True, out=None):
    """conv_forward after the inputs in `state` [B, K-1, D] (x's type, oldest
    first), which is replaced by the last K-1 inputs."""
    if state is None:
        raise ValueError("conv_prefill needs a state")
    return _conv(x, weight, bias, silu, state, out, 3)


def conv_step(state, x_t, weight, bias=None, silu=True, out=None):
    """One token a sequence: x_t [B, D] -> [B, D]; `state` as in conv_prefill."""
    if state is None:
        raise ValueError("conv_step needs a state")
    return _conv(x_t, weight, bias, silu, state, out, 2)


def conv_backward(x, weight, bias, dy, silu=True):
    """Gradients (dx, dweight, dbias or None) of conv_forward for dy [B, n, D]."""
    D, K, code, wcode = _conv_args(x, weight, bias, 3)
    B, n = x.shape[:2]
    _same("dy", dy, x.shape, x.dtype, x.device)
    rows, grows = _rows("x", x, 1), _rows("dy", dy, 1)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    ws, nb = _space(capi.hla_conv_backward_workspace_bytes(B, n, D, K), x.device)
    _launch(capi.hla_conv_backward, x, *rows, weight.data_ptr(), _ptr(bias), *grows, dx.data_ptr(), dw.data_ptr(),
            _ptr(db), B, n, D, K, int(bool(silu)), code, wcode, ws.data_ptr(), nb)
    return dx, dw, db


class ShortConv(torch.autograd.Function):
    """conv_forward as a differentiable op."""

    @staticmethod
    def forward(ctx, x, weight, bias, silu):
        ctx.save_for_backward(x, weight, bias)
        ctx.silu = silu
        return conv_forward(x, weight, bias, silu)

    @staticmethod
    @once
    def backward(ctx, dy):
        x, weight, bias = ctx.saved_tensors
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        return (*conv_backward(x, weight, bias, dy, ctx.silu), None)


def short_conv(x, weight, bias=None, silu=True):
    """Differentiable conv_forward."""
    if not _learns(x, weight, bias):
        return conv_forward(x, weight, bias, silu)
    return ShortConv.apply(x, weight, bias, silu)


# ----------------------------------------------------------------------------
# Norm and rotation of queries and keys
def _qk_args(q, k, q_weight, k_weight, cos, sin, positions):
    """The sizes and codes of a call, and its leading C arguments."""
    for name, t in (("q", q), ("k", k)):
        if t.dim() != 4:
            raise ValueError(f"{name} must have 4 dimensions [B, n, heads, d], got shape {tuple(t.shape)}")
    B, n, H, d = q.shape
    Hk = k.shape[2]
    _same("k", k, (B, n, Hk, d), q.dtype, q.device)
    weights = [w for w in (q_weight, k_weight) if w is not None]
    wtype = weights[0].dtype if weights else q.dtype
    _same("q_weight", q_weight, (d,), wtype, q.device, contiguous=True)
    _same("k_weight", k_weight, (d,), wtype, q.device, contiguous=True)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    rot, count = 0, 0
    if cos is not None:
        if cos.dim() != 2:
            raise ValueError(f"cos must be [positions, rot / 2], got {tuple(cos.shape)}")
        _same("cos", cos, cos.shape, torch.float32, q.device, contiguous=True)
        _same("sin", sin, cos.shape, torch.float32, q.device, contiguous=True)
        count, rot = cos.shape[0], 2 * cos.shape[1]
    pos_bs, pos64 = 0, 0
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"positions must be int32 or int64, got {positions.dtype}")
        _same("positions", positions, (n,) if positions.dim() == 1 else (B, n), None, q.device)
        if n != 1 and positions.stride(-1) != 1:
            raise ValueError("positions: the last dimension must be contiguous")
        pos_bs = positions.stride(0) if positions.dim() == 2 and B != 1 else 0
        pos64 = int(positions.dtype == torch.int64)
    _on_gpu(q)
    code, wcode = _code("q", q), _CODES.get(wtype)
    if wcode is None:
        raise TypeError(f"weights must be float32 or bfloat16, got {wtype}")
    lead = (*_rows("q", q, 2), *_rows("k", k, 2), _ptr(q_weight), _ptr(k_weight), _ptr(cos), _ptr(sin),
            _ptr(positions), pos_bs)
    return lead, (B, n, H, Hk, d, rot, count), (code, wcode, pos64)


def qk_norm_rope_forward(q, k, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, eps=1e-6,
                         interleaved=False):
    """Norm and rotation of every head of q [B, n, H, d] and k [B, n, Hk, d],
    laid out for the attention: ([B, H, n, d], [B, Hk, n, d]).  Each head's
    row becomes weight x / sqrt(mean(x^2) + eps) and its first 2 cos.shape[1]
    dimensions turn by the angles in row positions[b, t] (default t) of the
    fp32 tables cos and sin: halves of a pair rot/2 apart, or neighbours
    (interleaved).  weight = d^-0.5 gives rows of unit length.  A position
    outside the tables gives NaN."""
    lead, sizes, codes = _qk_args(q, k, q_weight, k_weight, cos, sin, positions)
    B, n, H, Hk, d = sizes[:5]
    qo = torch.empty((B, H, n, d), dtype=q.dtype, device=q.device)
    ko = torch.empty((B, Hk, n, d), dtype=q.dtype, device=q.device)
    _launch(capi.hla_qk_norm_rope, q, *lead, qo.data_ptr(), ko.data_ptr(), *sizes, int(bool(interleaved)),
            float(eps), *codes)
    return qo, ko


def qk_norm_rope_backward(q, k, q_weight, k_weight, cos, sin, positions, dq_out, dk_out, eps=1e-6, interleaved=False):
    """Gradients (dq, dk, dq_weight, dk_weight) of qk_norm_rope_forward for
    dq_out [B, H, n, d] and dk_out [B, Hk, n, d]; None for a weight not given."""
    lead, sizes, codes = _qk_args(q, k, q_weight, k_weight, cos, sin, positions)
    B, n, H, Hk, d = sizes[:5]
    _same("dq_out", dq_out, (B, H, n, d), q.dtype, q.device, contiguous=True)
    _same("dk_out", dk_out, (B, Hk, n, d), q.dtype, q.device, contiguous=True)
    dq = torch.empty((B, n, H, d), dtype=q.dtype, device=q.device)
    dk = torch.empty((B, n, Hk, d), dtype=q.dtype, device=q.device)
    dqw, dkw = (None if w is None else torch.empty_like(w) for w in (q_weight, k_weight))
    ws, nb = _space(capi.hla_qk_norm_rope_backward_workspace_bytes(d), q.device)
    _launch(capi.hla_qk_norm_rope_backward, q, *lead, dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(),
            dk.data_ptr(), _ptr(dqw), _ptr(dkw), *sizes, int(bool(interleaved)), float(eps), *codes, ws.data_ptr(),
            nb)
    return dq, dk, dqw, dkw


class QKNormRope(torch.autograd.Function):
    """qk_norm_rope_forward as a differentiable op."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.how = eps, interleaved
        return qk_norm_rope_forward(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)

    @staticmethod
    @once
    def backward(ctx, dq_out, dk_out):
        grads = qk_norm_rope_backward(*ctx.saved_tensors, _upstream(dq_out), _upstream(dk_out), *ctx.how)
        return (*grads, None, None, None, None, None)


def qk_norm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, eps=1e-6, interleaved=False):
    """Differentiable qk_norm_rope_forward (in q, k and the weights)."""
    if not _learns(q, k, q_weight, k_weight):
        return qk_norm_rope_forward(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    return QKNormRope.apply(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)


# ----------------------------------------------------------------------------
# Selective state space scan
def _ssm_args(x, dt, A, Bm, Cm, D, dt_bias, step=False):
    """(rows of x, dt, Bm, Cm; B, n, H, P, G, N; codes), checked."""
    rank = 3 if step else 4
    for name, t in (("x", x), ("Bm", Bm), ("Cm", Cm)):
        if t.dim() != rank:
            raise ValueError(f"{name} must have {rank} dimensions, got shape {tuple(t.shape)}")
    H, P = x.shape[-2:]
    G, N = Bm.shape[-2:]
    lead = tuple(x.shape[:-2])
    _same("dt", dt, (*lead, H), None, x.device)
    _same("Bm", Bm, (*lead, G, N), x.dtype, x.device)
    _same("Cm", Cm, (*lead, G, N), x.dtype, x.device)
    for name, t in (("A", A), ("D", D), ("dt_bias", dt_bias)):
        _same(name, t, (H,), torch.float32, x.device, contiguous=True)
    _on_gpu(x)
    codes = _code("x", x), _code("dt", dt)
    rows = _rows("x", x, 2), _rows("dt", dt, 1), _rows("Bm", Bm, 2), _rows("Cm", Cm, 2)
    return rows, (lead[0], 1 if step else lead[1], H, P, G, N), codes


def _ssm(state, x, dt, A, Bm, Cm, D, dt_bias, softplus, out, workspace):
    (rx, rt, rb, rc), sizes, codes = _ssm_args(x, dt, A, Bm, Cm, D, dt_bias)
    B, n, H, P, G, N = sizes
    _same("state", state, (B, H, N, P), torch.float32, x.device, contiguous=True)
    out = _out(out, x.shape, x)
    ws, nb = _space(capi.hla_ssm_workspace_bytes(*sizes, codes[0]), x.device, workspace)
    _launch(capi.hla_ssm_forward, x, *rx, *rt, A.data_ptr(), *rb, *rc, _ptr(D), _ptr(dt_bias), _ptr(state),
            out.data_ptr(), *sizes, int(bool(softplus)), *codes, ws.data_ptr(), nb)
    return out


def ssm_forward(x, dt, A, Bm, Cm, D=None, dt_bias=None, softplus=True, out=None, workspace=None):
    """Selective state space scan from a zero state: x [B, n, H, P], dt
    [B, n, H], A, D, dt_bias fp32 [H], Bm, Cm [B, n, G, N] (G divides H) -> y
    [B, n, H, P] of x's type.  With dt = softplus(dt + dt_bias):
    h_t = exp(dt_t A) h_{t-1} + dt_t Bm_t x_t^T, y_t = h_t^T Cm_t + D x_t."""
    return _ssm(None, x, dt, A, Bm, Cm, D, dt_bias, softplus, out, workspace)


def ssm_prefill(state, x, dt, A, Bm, Cm, D=None, dt_bias=None, softplus=True, out=None, workspace=None):
    """ssm_forward from `state` (fp32 [B, H, N, P]), which becomes the state
    after the last token."""
    if state is None:
        raise ValueError("ssm_prefill needs a state")
    return _ssm(state, x, dt, A, Bm, Cm, D, dt_bias, softplus, out, workspace)


def ssm_step(state, x_t, dt_t, A, B_t, C_t, D=None, dt_bias=None, softplus=True, out=None):
    """One token a sequence: x_t [B, H, P], dt_t [B, H], B_t, C_t [B, G, N] -> [B, H, P]; `state` updated in place."""
    (rx, rt, rb, rc), (B, _, H, P, G, N), codes = _ssm_args(x_t, dt_t, A, B_t, C_t, D, dt_bias, step=True)
    if state is None:
        raise ValueError("ssm_step needs a state")
    _same("state", state, (B, H, N, P), torch.float32, x_t.device, contiguous=True)
    out = _out(out, x_t.shape, x_t)
    _launch(capi.hla_ssm_step, x_t, state.data_ptr(), *rx[:2], *rt[:2], A.data_ptr(), *rb[:2], *rc[:2], _ptr(D),
            _ptr(dt_bias), out.data_ptr(), B, H, P, G, N, int(bool(softplus)), *codes)
    return out


def ssm_backward(x, dt, A, Bm, Cm, D, dt_bias, dy, softplus=True):
    """Gradients (dx, ddt, dA, dBm, dCm, dD, ddt_bias) of ssm_forward for dy
    [B, n, H, P], bf16 inputs; None for a D or dt_bias not given."""
    (rx, rt, rb, rc), sizes, codes = _ssm_args(x, dt, A, Bm, Cm, D, dt_bias)
    _same("dy", dy, x.shape, x.dtype, x.device)
    ry = _rows("dy", dy, 2)
    dx, ddt, dB, dC = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (x, dt, Bm, Cm))
    dA, dD, db = (None if t is None else torch.empty_like(t) for t in (A, D, dt_bias))
    ws, nb = _space(capi.hla_ssm_backward_workspace_bytes(*sizes, codes[0]), x.device)
    _launch(capi.hla_ssm_backward, x, *rx, *rt, A.data_ptr(), *rb, *rc, _ptr(D), _ptr(dt_bias), *ry, dx.data_ptr(),
            ddt.data_ptr(), dA.data_ptr(), dB.data_ptr(), dC.data_ptr(), _ptr(dD), _ptr(db), *sizes,
            int(bool(softplus)), *codes, ws.data_ptr(), nb)
    return dx, ddt, dA, dB, dC, dD, db


class SSMScan(torch.autograd.Function):
    """ssm_forward as a differentiable op (bf16 inputs)."""

    @staticmethod
    def forward(ctx, x, dt, A, Bm, Cm, D, dt_bias, softplus):
        ctx.save_for_backward(x, dt, A, Bm, Cm, D, dt_bias)
        ctx.softplus = softplus
        return ssm_forward(x, dt, A, Bm, Cm, D, dt_bias, softplus)

    @staticmethod
    @once
    def backward(ctx, dy):
        return (*ssm_backward(*ctx.saved_tensors, _upstream(dy), ctx.softplus), None)


def ssm_scan(x, dt, A, Bm, Cm, D=None, dt_bias=None, softplus=True):
    """Differentiable ssm_forward.  The gradients cover bf16 inputs: fp32 ones
    that need them are refused here."""
    if x.dtype != torch.bfloat16 and _has_graph(x, dt, A, Bm, Cm, D, dt_bias):
        raise capi.HLAError(capi.HLA_ERR_UNSUPPORTED, "the scan's gradients cover bf16 inputs: x, Bm and Cm must be "
                            f"bf16 to be differentiated, got {x.dtype}; without gradients take ssm_forward or no_grad")
    if not _learns(x, dt, A, Bm, Cm, D, dt_bias):
        return ssm_forward(x, dt, A, Bm, Cm, D, dt_bias, softplus)
    return SSMScan.apply(x, dt, A, Bm, Cm, D, dt_bias, softplus)
