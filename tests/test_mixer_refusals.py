"""What the operators around the attention refuse, without a GPU: the C entry
points check sizes, flags, strides and pointers on the host before any device
call, and the torch binding checks shapes, types and layouts before them."""
import pytest
import torch

from paper_2510_27258_amd import capi, mixer

FP32, BF16 = capi.HLA_FP32, capi.HLA_BF16
INVALID, UNSUP, WORKSPACE = capi.HLA_ERR_INVALID, capi.HLA_ERR_UNSUPPORTED, capi.HLA_ERR_WORKSPACE
P = 256            # aligned and never dereferenced


def _refused(rc, code, text):
    assert rc == code, (rc, capi.hla_last_error())
    assert text in capi.hla_last_error(), capi.hla_last_error()


def _conv(**kw):
    a = dict(x=P, xb=0, xt=64, w=P, b=None, st=None, y=None, B=1, n=8, D=64, K=4, silu=1, dt=BF16, wdt=BF16)
    a.update(kw)
    return capi.lib().hla_conv_forward(a["x"], a["xb"], a["xt"], a["w"], a["b"], a["st"], a["y"], a["B"], a["n"], a["D"],
                                       a["K"], a["silu"], a["dt"], a["wdt"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(B=0), INVALID, "B, n and D"), (dict(n=0), INVALID, "B, n and D"), (dict(D=0), INVALID, "B, n and D"),
    (dict(K=1), UNSUP, "K must be"), (dict(K=5), UNSUP, "K must be"), (dict(B=65536), UNSUP, "65535"),
    (dict(n=(1 << 22) + 1), UNSUP, "2^22"), (dict(n=1 << 22, D=1 << 20), UNSUP, "too long"),
    (dict(silu=2), INVALID, "silu"), (dict(dt=2), INVALID, "dtype"), (dict(wdt=-1), INVALID, "w_dtype"),
    (dict(x=None), INVALID, "x is NULL"), (dict(x=P + 1), INVALID, "x is not 2-byte"), (dict(xt=-1), INVALID, "strides"),
    (dict(w=None), INVALID, "weight is NULL"), (dict(b=P + 1), INVALID, "bias is not"), (dict(), INVALID, "y is NULL"),
    (dict(y=P, st=P + 1), INVALID, "state is not")])
def test_conv_forward(kw, code, text):
    _refused(_conv(**kw), code, text)


def test_conv_backward():
    L = capi.lib()

    def call(dy=P, dx=P, dw=P, ws=P, nb=1 << 30, K=4):
        return L.hla_conv_backward(P, 0, 64, P, None, dy, 0, 64, dx, dw, None, 1, 8, 64, K, 1, BF16, BF16, ws, nb, None)
    _refused(call(dy=None), INVALID, "dy is NULL")
    _refused(call(dx=None), INVALID, "dx is NULL")
    _refused(call(dw=None), INVALID, "dweight is NULL")
    _refused(call(ws=None), WORKSPACE, "workspace of")
    _refused(call(nb=16), WORKSPACE, "workspace of")
    _refused(call(ws=P + 4), INVALID, "workspace is not 16-byte")
    _refused(call(K=7), UNSUP, "K must be")
    assert capi.hla_conv_backward_workspace_bytes(1, 0, 8, 4) == 0
    assert capi.hla_conv_backward_workspace_bytes(1, 8, 8, 4) > 0


def _qk(**kw):
    a = dict(q=P, qb=0, qt=256, k=P, kt=256, qw=P, cos=P, sin=P, pos=P, pb=0, qo=P, ko=None, B=1, n=8, H=2, Hk=2, d=128,
             rot=128, cnt=100, il=0, eps=1e-6, dt=BF16, wdt=BF16, p64=1)
    a.update(kw)
    return capi.lib().hla_qk_norm_rope(a["q"], a["qb"], a["qt"], a["k"], 0, a["kt"], a["qw"], None, a["cos"], a["sin"],
                                       a["pos"], a["pb"], a["qo"], a["ko"], a["B"], a["n"], a["H"], a["Hk"], a["d"],
                                       a["rot"], a["cnt"], a["il"], a["eps"], a["dt"], a["wdt"], a["p64"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(B=0), INVALID, "B, n, H and Hk"), (dict(n=-1), INVALID, "B, n, H and Hk"), (dict(Hk=0), INVALID, "B, n, H"),
    (dict(d=12), UNSUP, "d must be"), (dict(d=264), UNSUP, "d must be"), (dict(d=100), UNSUP, "d must be"),
    (dict(rot=130), INVALID, "rot must be"), (dict(rot=7), INVALID, "rot must be"), (dict(rot=-2), INVALID, "rot must"),
    (dict(cnt=0), INVALID, "positions"), (dict(il=3), INVALID, "interleaved"), (dict(eps=-1.0), INVALID, "eps"),
    (dict(eps=float("nan")), INVALID, "eps"), (dict(dt=3), INVALID, "dtype"), (dict(p64=2), INVALID, "pos64"),
    (dict(B=1 << 15, n=1 << 20, H=64), UNSUP, "too many rows"), (dict(q=None), INVALID, "q is NULL"),
    (dict(q=P + 8), INVALID, "q is not 16-byte"), (dict(qt=260), INVALID, "whole 16-byte"),
    (dict(kt=-8), INVALID, "strides"), (dict(qw=P + 1), INVALID, "q_weight"), (dict(cos=None), INVALID, "cos is NULL"),
    (dict(sin=P + 2), INVALID, "sin is not"), (dict(pos=P + 4), INVALID, "pos is not 8-byte"),
    (dict(pb=-1), INVALID, "pos_bs"), (dict(qo=None), INVALID, "q_out is NULL"), (dict(), INVALID, "k_out is NULL")])
def test_qk_norm_rope(kw, code, text):
    _refused(_qk(**kw), code, text)


def test_qk_norm_rope_backward():
    L = capi.lib()

    def call(gq=P, dk=P, ws=P, nb=1 << 30):
        return L.hla_qk_norm_rope_backward(P, 0, 256, P, 0, 256, P, P, P, P, P, 0, gq, P, P, dk, P, P, 1, 8, 2, 2, 128,
                                           128, 100, 0, 1e-6, BF16, BF16, 1, ws, nb, None)
    _refused(call(gq=None), INVALID, "dq_out is NULL")
    _refused(call(dk=P + 2), INVALID, "dk is not 16-byte")
    _refused(call(nb=64), WORKSPACE, "workspace of")
    assert capi.hla_qk_norm_rope_backward_workspace_bytes(20) == 0
    assert capi.hla_qk_norm_rope_backward_workspace_bytes(64) > 0


def _ssm(**kw):
    a = dict(x=P, xt=128, dt=P, dtt=2, A=P, b=P, bt=64, c=P, D=None, bias=None, st=None, y=None, B=1, n=8, H=2, P=64, G=1,
             N=64, soft=1, ty=BF16, dty=BF16, ws=P, nb=1 << 40)
    a.update(kw)
    return capi.lib().hla_ssm_forward(a["x"], 0, a["xt"], a["dt"], 0, a["dtt"], a["A"], a["b"], 0, a["bt"], a["c"], 0, 64,
                                      a["D"], a["bias"], a["st"], a["y"], a["B"], a["n"], a["H"], a["P"], a["G"], a["N"],
                                      a["soft"], a["ty"], a["dty"], a["ws"], a["nb"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(n=0), INVALID, "B, n, H and G"), (dict(G=0), INVALID, "B, n, H and G"), (dict(H=3, G=2), INVALID, "multiple of"),
    (dict(B=300, H=300), UNSUP, "65535"), (dict(P=24), UNSUP, "P and N"), (dict(N=144), UNSUP, "P and N"),
    (dict(P=8), UNSUP, "P and N"), (dict(B=64, H=512, n=1 << 16), UNSUP, "too long"), (dict(soft=2), INVALID, "softplus"),
    (dict(ty=5), INVALID, "dtype"), (dict(dty=5), INVALID, "dt_dtype"), (dict(x=None), INVALID, "x is NULL"),
    (dict(x=P + 8), INVALID, "x is not 16-byte"), (dict(xt=129), INVALID, "whole 16-byte"),
    (dict(xt=1 << 28), UNSUP, "too long"), (dict(b=P + 2), INVALID, "Bm is not"), (dict(bt=4), INVALID, "whole 16-byte"),
    (dict(c=None), INVALID, "Cm is NULL"), (dict(dt=P + 1), INVALID, "dt is not"), (dict(dtt=-2), INVALID, "strides"),
    (dict(A=None), INVALID, "A is NULL"), (dict(D=P + 2), INVALID, "D is not"), (dict(bias=P + 1), INVALID, "dt_bias"),
    (dict(), INVALID, "y is NULL"), (dict(y=P, st=P + 8), INVALID, "state is not"),
    (dict(y=P, ws=None), WORKSPACE, "workspace of"), (dict(y=P, nb=128), WORKSPACE, "workspace of")])
def test_ssm_forward(kw, code, text):
    _refused(_ssm(**kw), code, text)


def test_ssm_step_and_backward():
    L = capi.lib()
    _refused(L.hla_ssm_step(None, P, 0, P, 0, P, P, 0, P, 0, None, None, P, 1, 2, 64, 1, 64, 1, BF16, BF16, None), INVALID,
             "state is NULL")
    _refused(L.hla_ssm_step(P, P, 0, P, 0, P, P, 0, P, 0, None, None, P, 1, 2, 60, 1, 64, 1, BF16, BF16, None), UNSUP, "P and N")

    def back(ty=BF16, dy=P, dA=P, nb=1 << 40):
        return L.hla_ssm_backward(P, 0, 128, P, 0, 2, P, P, 0, 64, P, 0, 64, None, None, dy, 0, 128, P, P, dA, P, P, None,
                                  None, 1, 8, 2, 64, 1, 64, 1, ty, BF16, P, nb, None)
    _refused(back(ty=FP32), UNSUP, "bf16")
    _refused(back(dy=None), INVALID, "dy is NULL")
    _refused(back(dA=None), INVALID, "dA is NULL")
    _refused(back(nb=0), WORKSPACE, "workspace of")
    assert capi.hla_ssm_workspace_bytes(1, 8, 2, 60, 1, 64, BF16) == 0
    assert capi.hla_ssm_workspace_bytes(1, 8, 2, 64, 1, 64, FP32) > 0
    assert capi.hla_ssm_backward_workspace_bytes(1, 8, 2, 64, 1, 64, FP32) == 0
    assert capi.hla_ssm_backward_workspace_bytes(1, 8, 2, 64, 1, 64, BF16) > 0


# ----------------------------------------------------------------------------
# The binding: each case fails on its own mismatch, before the check for a GPU.
def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def _rejects(error, f, text):
    with pytest.raises(error) as e:
        f()
    assert text in str(e.value) and "GPU" not in str(e.value), str(e.value)


def test_binding_conv():
    x, w = _z(2, 8, 16), _z(16, 4)
    _rejects(ValueError, lambda: mixer.conv_forward(x[0], w), "3 dimensions")
    _rejects(ValueError, lambda: mixer.conv_forward(x, _z(8, 4)), "weight must be")
    _rejects(ValueError, lambda: mixer.conv_forward(x, _z(4, 16).t()), "weight must be contiguous")
    _rejects(ValueError, lambda: mixer.conv_forward(x, w, _z(8)), "bias must be")
    _rejects(ValueError, lambda: mixer.conv_forward(x, w, _z(16, dtype=torch.float32)), "bias must be")
    _rejects(ValueError, lambda: mixer.conv_prefill(None, x, w), "needs a state")
    with pytest.raises(ValueError, match="GPU"):
        mixer.conv_forward(x, w)


def test_binding_qk():
    q, k = _z(2, 8, 4, 64), _z(2, 8, 2, 64)
    t = _z(8, 32, dtype=torch.float32)
    call = mixer.qk_norm_rope_forward
    _rejects(ValueError, lambda: call(q[0], k), "4 dimensions")
    _rejects(ValueError, lambda: call(q, _z(2, 8, 2, 32)), "k must be")
    _rejects(ValueError, lambda: call(q, k.float()), "k must be")
    _rejects(ValueError, lambda: call(q, k, _z(32)), "q_weight")
    _rejects(ValueError, lambda: call(q, k, _z(64), _z(64, dtype=torch.float32)), "k_weight")
    _rejects(ValueError, lambda: call(q, k, cos=t), "together")
    _rejects(ValueError, lambda: call(q, k, cos=t, sin=t[:4]), "sin")
    _rejects(ValueError, lambda: call(q, k, cos=t.bfloat16(), sin=t.bfloat16()), "cos")
    _rejects(ValueError, lambda: call(q, k, cos=t, sin=t, positions=_z(2, 8)), "positions must be int")
    _rejects(ValueError, lambda: call(q, k, cos=t, sin=t, positions=torch.zeros(2, 7, dtype=torch.int64)), "positions")
    with pytest.raises(ValueError, match="GPU"):
        call(q, k, cos=t, sin=t)


def test_binding_ssm():
    f = torch.float32
    good = dict(x=_z(2, 8, 4, 16), dt=_z(2, 8, 4), A=_z(4, dtype=f), Bm=_z(2, 8, 2, 16), Cm=_z(2, 8, 2, 16))

    def call(**kw):
        return lambda: mixer.ssm_forward(**{**good, **kw})
    _rejects(ValueError, call(x=_z(8, 4, 16)), "4 dimensions")
    _rejects(ValueError, call(dt=_z(2, 8, 3)), "dt must be")
    _rejects(ValueError, call(A=_z(4)), "A must be")
    _rejects(ValueError, call(D=_z(3, dtype=f)), "D must be")
    _rejects(ValueError, call(Cm=_z(2, 8, 2, 32)), "Cm must be")
    _rejects(ValueError, call(Bm=_z(2, 8, 2, 16, dtype=f)), "Bm must be")
    _rejects(ValueError, lambda: mixer.ssm_prefill(None, **good), "needs a state")
    with pytest.raises(ValueError, match="GPU"):
        call()()


def test_rows_need_contiguous_tokens():
    assert mixer._rows("x", _z(3, 5, 2, 8)[:, ::2], 2)[1:] == (80, 32)
    assert mixer._rows("x", _z(1, 1, 2, 8)[:, :1], 2)[1:] == (0, 0)
    with pytest.raises(ValueError):
        mixer._rows("x", _z(3, 2, 5, 8).transpose(1, 2), 2)
    with pytest.raises(ValueError):
        mixer._rows("x", _z(3, 5, 16)[..., ::2], 1)
