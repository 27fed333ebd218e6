"""What the operators of a block refuse, without a GPU: the C entry points check
sizes, flags, strides, pointers and workspaces on the host before any device
call, and the torch binding checks shapes, types and layouts before them."""
import math

import pytest
import torch

from paper_2510_27258_amd import block, capi

FP32, BF16 = capi.HLA_FP32, capi.HLA_BF16
INVALID, UNSUP, WORKSPACE = capi.HLA_ERR_INVALID, capi.HLA_ERR_UNSUPPORTED, capi.HLA_ERR_WORKSPACE
P = 256            # aligned and never dereferenced


def _refused(rc, code, text):
    assert rc == code, (rc, capi.hla_last_error())
    assert text in capi.hla_last_error(), capi.hla_last_error()


def _gn(back=False, **kw):
    a = dict(y=P, yb=0, yt=256, yg=64, z=P, zb=0, zt=256, zg=64, w=P, out=None, B=1, n=8, G=4, d=64, per=0, first=0, eps=1e-6,
             ydt=BF16, dt=BF16, wdt=BF16, dy=P, dyb=0, dyt=256, dyg=64, dz=P, dw=P, ws=None, nb=0)
    a.update(kw)
    lead = (a["y"], a["yb"], a["yt"], a["yg"], a["z"], a["zb"], a["zt"], a["zg"], a["w"], a["out"])
    sizes = (a["B"], a["n"], a["G"], a["d"], a["per"], a["first"], a["eps"], a["ydt"], a["dt"], a["wdt"])
    if back:
        return capi.lib().hla_gated_norm_backward(*lead, a["dy"], a["dyb"], a["dyt"], a["dyg"], a["dz"], a["dw"], *sizes, a["ws"],
                                                  a["nb"], None)
    return capi.lib().hla_gated_norm(*lead, *sizes, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(B=0), INVALID, "B and n"), (dict(n=0), INVALID, "B and n"), (dict(G=0), INVALID, "G and d"), (dict(d=0), INVALID, "G and d"),
    (dict(B=1 << 16, n=1 << 15), UNSUP, "2^31"), (dict(d=16385), UNSUP, "16384"), (dict(G=65536), UNSUP, "65535"),
    (dict(per=2), INVALID, "per_group"), (dict(first=-1), INVALID, "norm_first"), (dict(eps=-1e-6), INVALID, "eps"),
    (dict(eps=math.inf), INVALID, "eps"), (dict(eps=math.nan), INVALID, "eps"), (dict(ydt=2), INVALID, "y_dtype"),
    (dict(dt=-1), INVALID, "dtype"), (dict(dt=FP32), UNSUP, "bf16 beside fp32"), (dict(wdt=5), INVALID, "w_dtype"),
    (dict(y=None), INVALID, "y is NULL"), (dict(y=P + 1), INVALID, "y is not 2-byte"), (dict(y=P + 2, ydt=FP32), INVALID, "y is not 4-byte"),
    (dict(yt=-1), INVALID, "y: strides"), (dict(z=P + 1), INVALID, "z is not"), (dict(zg=-64), INVALID, "z: strides"),
    (dict(w=P + 1), INVALID, "weight is not"), (dict(), INVALID, "out is NULL"), (dict(out=P + 1), INVALID, "out is not")])
def test_gated_norm(kw, code, text):
    _refused(_gn(**kw), code, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(), INVALID, "dout is NULL"), (dict(out=P, dy=None), INVALID, "dy is NULL"), (dict(out=P, dz=None), INVALID, "dz is NULL"),
    (dict(out=P, z=None, dz=None), WORKSPACE, "workspace of"), (dict(out=P, dyg=63), INVALID, "overlap"),
    (dict(out=P, dyt=0), INVALID, "overlap"), (dict(out=P, B=2, dyb=0), INVALID, "overlap"), (dict(out=P, dw=P + 1), INVALID, "dweight"),
    (dict(out=P), WORKSPACE, "workspace of"), (dict(out=P, ws=P, nb=64), WORKSPACE, "workspace of"),
    (dict(out=P, ws=P + 4, nb=1 << 30), INVALID, "workspace is not 16-byte"), (dict(out=P, d=16385), UNSUP, "16384")])
def test_gated_norm_backward(kw, code, text):
    _refused(_gn(True, **kw), code, text)
    assert capi.hla_gated_norm_backward_workspace_bytes(1, 8, 4, 0, 0) == 0
    assert capi.hla_gated_norm_backward_workspace_bytes(1, 8, 4, 64, 1) > 0


def _rn(back=False, **kw):
    a = dict(x=P, xb=0, xt=64, y=P, yb=0, yt=64, w=P, post=P, scale=P, a0=None, a1=None, B=1, n=8, D=64, alpha=1.0, eps=1e-6, xdt=BF16,
             dt=BF16, wdt=BF16, dx=P, dy=P, dw=P, dpost=P, dscale=P, ws=None, nb=0)
    a.update(kw)
    lead = (a["x"], a["xb"], a["xt"], a["y"], a["yb"], a["yt"], a["w"], a["post"], a["scale"], a["a0"], a["a1"])
    sizes = (a["B"], a["n"], a["D"], a["alpha"], a["eps"], a["xdt"], a["dt"], a["wdt"])
    if back:
        return capi.lib().hla_residual_norm_backward(*lead, a["dx"], a["dy"], a["dw"], a["dpost"], a["dscale"], *sizes, a["ws"],
                                                     a["nb"], None)
    return capi.lib().hla_residual_norm(*lead, *sizes, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(B=0), INVALID, "B and n"), (dict(D=0), INVALID, "D must"), (dict(D=16385), UNSUP, "16384"), (dict(n=1 << 30, B=2), UNSUP, "2^31"),
    (dict(alpha=math.inf), INVALID, "alpha"), (dict(eps=-1.0), INVALID, "eps"), (dict(dt=FP32), UNSUP, "bf16 beside fp32"),
    (dict(wdt=2), INVALID, "w_dtype"), (dict(x=None), INVALID, "x is NULL"), (dict(y=P + 1), INVALID, "y is not"),
    (dict(xt=-64), INVALID, "x: strides"), (dict(post=P + 1), INVALID, "post_weight"), (dict(scale=P + 1), INVALID, "scale"),
    (dict(), INVALID, "out is NULL"), (dict(a0=P), INVALID, "r is NULL")])
def test_residual_norm(kw, code, text):
    _refused(_rn(**kw), code, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(), INVALID, "dout is NULL"), (dict(a0=P, dx=None), INVALID, "dx is NULL"), (dict(a1=P, dy=None), INVALID, "dy is NULL"),
    (dict(a0=P, post=None), INVALID, "without a post_weight"), (dict(a0=P, dscale=P + 1), INVALID, "dscale"),
    (dict(a1=P), WORKSPACE, "workspace of"), (dict(a0=P, ws=P, nb=16), WORKSPACE, "workspace of")])
def test_residual_norm_backward(kw, code, text):
    _refused(_rn(True, **kw), code, text)
    assert capi.hla_residual_norm_backward_workspace_bytes(1, 8, 16385) == 0
    assert capi.hla_residual_norm_backward_workspace_bytes(1, 8, 64) > 0


def _glr(kind="forward", **kw):
    a = dict(x=P, xb=0, xt=64, f=P, ft=64, g=P, gt=64, decay=P, fb=P, gb=P, state=None, y=None, kept=None, B=1, n=8, D=64, c=8.0, dt=BF16,
             ws=None, nb=0, dy=P, dyt=64, dx=P, df=P, dg=P, dd=P, dfb=P, dgb=P)
    a.update(kw)
    rows = (a["x"], a["xb"], a["xt"], a["f"], 0, a["ft"], a["g"], 0, a["gt"])
    params = (a["decay"], a["fb"], a["gb"])
    if kind == "step":
        return capi.lib().hla_glr_step(a["state"], a["x"], a["xb"], a["f"], 64, a["g"], 64, *params, a["y"], a["B"], a["D"], a["c"],
                                       a["dt"], None)
    if kind == "backward":
        return capi.lib().hla_glr_backward(*rows, *params, a["kept"], a["dy"], 0, a["dyt"], a["dx"], a["df"], a["dg"], a["dd"], a["dfb"],
                                           a["dgb"], a["B"], a["n"], a["D"], a["c"], a["dt"], a["ws"], a["nb"], None)
    return capi.lib().hla_glr_forward(*rows, *params, a["state"], a["y"], a["kept"], a["B"], a["n"], a["D"], a["c"], a["dt"], a["ws"],
                                      a["nb"], None)


@pytest.mark.parametrize("kind", ["forward", "backward"])
@pytest.mark.parametrize("kw,code,text", [
    (dict(B=0), INVALID, "B and n"), (dict(n=0), INVALID, "B and n"), (dict(D=0), INVALID, "D must"), (dict(D=(1 << 21) + 1), UNSUP, "2^21"),
    (dict(B=1 << 12, n=1 << 19), UNSUP, "2^31"), (dict(B=1 << 14, D=1 << 21), UNSUP, "too many channels"), (dict(dt=3), INVALID, "dtype"),
    (dict(c=-1.0), INVALID, "c must"), (dict(c=math.nan), INVALID, "c must"), (dict(x=None), INVALID, "x is NULL"),
    (dict(f=P + 1), INVALID, "f is not"), (dict(gt=-2), INVALID, "g: strides"), (dict(ft=(1 << 21) + 1), UNSUP, "f: a token stride"),
    (dict(decay=None), INVALID, "decay is NULL"), (dict(fb=P + 2), INVALID, "f_bias"), (dict(gb=P + 2), INVALID, "g_bias")])
def test_recurrence(kind, kw, code, text):
    _refused(_glr(kind, **kw), code, text)


def test_recurrence_pointers_and_workspaces():
    _refused(_glr(), INVALID, "y is NULL")
    _refused(_glr(y=P, state=P + 2), INVALID, "state is not")
    _refused(_glr(y=P, kept=P + 2), INVALID, "kept is not")
    _refused(_glr(y=P), WORKSPACE, "workspace of")
    _refused(_glr(y=P, ws=P, nb=8), WORKSPACE, "workspace of")
    _refused(_glr("step"), INVALID, "y is NULL")
    _refused(_glr("step", y=P), INVALID, "state is NULL")
    _refused(_glr("backward"), INVALID, "kept is NULL")
    for name, text in (("dy", "dy is NULL"), ("dx", "dx is NULL"), ("df", "df is NULL"), ("dg", "dg is NULL"), ("dd", "ddecay is NULL")):
        _refused(_glr("backward", kept=P, **{name: None}), INVALID, text)
    _refused(_glr("backward", kept=P, dyt=(1 << 21) + 1), UNSUP, "dy: a token stride")
    _refused(_glr("backward", kept=P), WORKSPACE, "workspace of")
    for query in (capi.hla_glr_workspace_bytes, capi.hla_glr_kept_bytes, capi.hla_glr_backward_workspace_bytes):
        assert query(1, 0, 64) == 0 and query(1, 8, 64) > 0
    assert capi.hla_glr_kept_bytes(2, 129, 3) == 2 * 2 * 3 * 4


def _glu(back=False, **kw):
    a = dict(x=P, xb=0, xt=64, wg=P, wu=P, h=None, B=1, n=8, D=64, F=128, act=0, dt=BF16, dh=P, dht=128, dx=P, dwg=P, dwu=P, ws=None, nb=0)
    a.update(kw)
    if back:
        return capi.lib().hla_glu_backward(a["x"], a["xb"], a["xt"], a["wg"], a["wu"], a["dh"], 0, a["dht"], a["dx"], a["dwg"], a["dwu"],
                                           a["B"], a["n"], a["D"], a["F"], a["act"], a["dt"], a["ws"], a["nb"], None)
    return capi.lib().hla_glu_forward(a["x"], a["xb"], a["xt"], a["wg"], a["wu"], a["h"], a["B"], a["n"], a["D"], a["F"], a["act"], a["dt"],
                                      None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code,text", [
    (dict(n=0), INVALID, "B and n"), (dict(D=0), INVALID, "D and F"), (dict(F=-8), INVALID, "D and F"), (dict(D=60), UNSUP, "multiples of 8"),
    (dict(F=130), UNSUP, "multiples of 8"), (dict(D=(1 << 20) + 8), UNSUP, "2^20"), (dict(n=1 << 22, F=1 << 20), UNSUP, "too many tiles"),
    (dict(B=1 << 20, n=2, F=1 << 15), UNSUP, "too many tiles"), (dict(D=1 << 20, F=1 << 20), UNSUP, "too many tiles"),
    (dict(act=2), INVALID, "act must"), (dict(dt=FP32), UNSUP, "cover bf16"), (dict(dt=7), INVALID, "dtype"),
    (dict(x=None), INVALID, "x is NULL"), (dict(x=P + 8), INVALID, "x is not 16-byte"), (dict(xt=60), INVALID, "16-byte pieces"),
    (dict(xt=1 << 22), UNSUP, "too long"), (dict(wg=P + 2), INVALID, "w_gate is not"), (dict(wu=None), INVALID, "w_up is NULL")])
def test_projections(back, kw, code, text):
    _refused(_glu(back, **kw), code, text)


def test_projections_of_many_short_sequences():
    """Sequences laid one behind the other are tiled as one; apart, each has tiles of its own."""
    many = dict(B=1 << 20, F=1 << 14)
    _refused(_glu(n=2, xb=128, **many), INVALID, "h is NULL")
    _refused(_glu(n=1, xb=72, **many), INVALID, "h is NULL")
    _refused(_glu(n=2, xb=192, **many), UNSUP, "laid apart")
    _refused(_glu(True, n=2, xb=128, dht=1 << 14, **many), UNSUP, "laid apart")       # dh's batches lie on one another
    assert capi.hla_glu_backward_workspace_bytes(1 << 20, 2, 64, 1 << 14) > 0


def test_projections_pointers_and_workspace():
    _refused(_glu(), INVALID, "h is NULL")
    _refused(_glu(h=P + 8), INVALID, "h is not 16-byte")
    for name, text in (("dh", "dh is NULL"), ("dx", "dx is NULL"), ("dwg", "dw_gate is NULL"), ("dwu", "dw_up is NULL")):
        _refused(_glu(True, **{name: None}), INVALID, text)
    _refused(_glu(True, dht=124), INVALID, "16-byte pieces")
    _refused(_glu(True), WORKSPACE, "workspace of")
    _refused(_glu(True, ws=P, nb=1 << 10), WORKSPACE, "workspace of")
    assert capi.hla_glu_backward_workspace_bytes(1, 8, 60, 128) == 0
    assert capi.hla_glu_backward_workspace_bytes(1, 8, 64, 128) > 0


# ----------------------------------------------------------------------------
# The torch binding
Z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)  # noqa: E731
H = torch.float16


@pytest.mark.parametrize("call,error,text", [
    (lambda: block.gated_norm(Z(2, 8, 64)), ValueError, "4 dimensions"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64), Z(2, 8, 4, 32)), ValueError, "z must be"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64), Z(2, 8, 4, 64), out_dtype=torch.float32), ValueError, "z must be torch.float32"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64), None, Z(4, 32)), ValueError, "weight must be"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64), None, Z(64, t=H)), TypeError, "weights must be"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64), None, Z(128)[::2]), ValueError, "contiguous"),
    (lambda: block.gated_norm(Z(2, 8, 4, 64, t=H)), ValueError, "GPU"),
    (lambda: block.residual_norm(Z(8, 64), Z(8, 64)), ValueError, "3 dimensions"),
    (lambda: block.residual_norm(Z(2, 8, 64), Z(2, 8, 32)), ValueError, "y must be"),
    (lambda: block.residual_norm(Z(2, 8, 64), Z(2, 8, 64), Z(64), Z(64, t=torch.float32)), ValueError, "post_weight must be"),
    (lambda: block.residual_norm(Z(2, 8, 64), Z(2, 8, 64), scale=Z(1)), ValueError, "scale must be"),
    (lambda: block.glr_forward(Z(2, 64), Z(2, 64), Z(2, 64), Z(64)), ValueError, "3 dimensions"),
    (lambda: block.glr_forward(Z(2, 8, 64), Z(2, 8, 64), Z(2, 8, 64, t=H), Z(64)), ValueError, "g must be"),
    (lambda: block.glr_forward(Z(2, 8, 64), Z(2, 8, 64), Z(2, 8, 64), Z(64)), ValueError, "decay must be torch.float32"),
    (lambda: block.glr_prefill(None, Z(2, 8, 64), Z(2, 8, 64), Z(2, 8, 64), Z(64, t=torch.float32)), ValueError, "needs a state"),
    (lambda: block.glu(Z(2, 64), Z(8, 64), Z(8, 64)), ValueError, "3 dimensions"),
    (lambda: block.glu(Z(2, 8, 64), Z(8, 32), Z(8, 32)), ValueError, "w_gate must be"),
    (lambda: block.glu(Z(2, 8, 64), Z(8, 64), Z(16, 64)), ValueError, "w_up must be"),
    (lambda: block.glu(Z(2, 8, 64), Z(64, 8).T, Z(8, 64)), ValueError, "contiguous"),
    (lambda: block.glu(Z(2, 8, 64), Z(8, 64, t=torch.float32), Z(8, 64)), ValueError, "w_gate must be torch.bfloat16"),
    (lambda: block.glu(Z(2, 8, 64), Z(8, 64), Z(8, 64), act="relu"), ValueError, "act must be"),
    (lambda: block.glu(Z(2, 8, 64), Z(8, 64), Z(8, 64)), ValueError, "GPU")])
def test_binding(call, error, text):
    with pytest.raises(error, match=text):
        call()


def test_binding_layouts(monkeypatch):
    monkeypatch.setattr(block, "_on_gpu", lambda t: None)
    monkeypatch.setattr(block, "_launch", lambda *a: None)
    with pytest.raises(ValueError, match="last dimension must be contiguous"):
        block.gated_norm(Z(2, 8, 64, 4).transpose(2, 3))
    with pytest.raises(ValueError, match="contiguous"):
        block.residual_norm(Z(2, 64, 8).transpose(1, 2), Z(2, 8, 64))
    with pytest.raises(ValueError, match="state must be"):
        block.glr_prefill(Z(2, 64), *(Z(2, 8, 64),) * 3, Z(64, t=torch.float32))
    with pytest.raises(ValueError, match="kept must be"):
        block.glr_backward(*(Z(2, 8, 64),) * 3, Z(64, t=torch.float32), None, None, Z(2, 8, 64), kept=Z(64, t=torch.float32))
    with pytest.raises(ValueError, match="needs a state"):
        block.glr_step(None, *(Z(2, 64),) * 3, Z(64, t=torch.float32))
    with pytest.raises(TypeError, match="must be float32 or bfloat16"):
        block.gated_norm(Z(2, 8, 4, 64, t=H))
    with pytest.raises(ValueError, match="dout must be contiguous"):
        block.gated_norm_backward(Z(2, 8, 4, 64), None, None, Z(2, 4, 8, 64).transpose(1, 2))
    # the stride of a dimension of one element is not looked at
    block.gated_norm(Z(2, 8, 4, 6)[..., :1])
