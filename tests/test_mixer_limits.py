"""Sizes that no launch of the operators around the attention can take, and
strides that are not used, at the C entry points, without a GPU: every such
size is refused on the host, before any kernel of the call."""
import pytest

from paper_2510_27258_amd import capi
from tests.test_mixer_refusals import BF16, FP32, INVALID, P, UNSUP, _conv, _qk, _refused, _ssm


# A launch has at most 2^32 threads.  Eight heads a thread: a token of H + Hk
# heads takes ceil(H / 8) + ceil(Hk / 8) rows of 16 lanes (bf16, d = 128).
@pytest.mark.parametrize("B,n,H,Hk,dtype,fits", [
    (1, (1 << 27) - 16, 1, 1, BF16, True), (1, 1 << 27, 1, 1, BF16, False), (1 << 10, 1 << 17, 1, 1, BF16, False),
    (1, (1 << 27) - 16, 8, 8, BF16, True), (1, 1 << 27, 8, 8, BF16, False),
    (1, 1 << 26, 8, 17, BF16, False), (1, (1 << 26) - 16, 8, 17, BF16, True),
    (1, (1 << 26) - 8, 1, 1, FP32, True), (1, 1 << 26, 1, 1, FP32, False)])
def test_qk_launches(B, n, H, Hk, dtype, fits):
    rc = _qk(B=B, n=n, H=H, Hk=Hk, qt=H * 128, kt=Hk * 128, dt=dtype)
    _refused(rc, *((INVALID, "k_out is NULL") if fits else (UNSUP, "too many rows")))


# The gradients' first launch has 512 threads for every 64 tokens, group and
# subset of a group's heads.
@pytest.mark.parametrize("B,n,H,G,fits", [
    (4, (1 << 23) - 64, 16, 16, True), (4, 1 << 23, 16, 16, False), (1, (1 << 25) + 1, 16, 16, False),
    (4, 1 << 24, 16, 8, False), (4, (1 << 24) - 64, 16, 8, True), (4, 1 << 24, 16, 1, True)])
def test_scan_gradient_launches(B, n, H, G, fits):
    need = capi.hla_ssm_backward_workspace_bytes(B, n, H, 16, G, 16, BF16)
    assert (need > 0) == fits
    if not fits:
        assert "too long" in capi.hla_last_error()
    rc = capi.lib().hla_ssm_backward(P, 0, H * 16, P, 0, H, P, P, 0, G * 16, P, 0, G * 16, None, None, P, 0, H * 16, P, P,
                                     P, P, P, None, None, B, n, H, 16, G, 16, 1, BF16, BF16, None, 0, None)
    _refused(rc, *((capi.HLA_ERR_WORKSPACE, "workspace of") if fits else (UNSUP, "too long")))


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_longest_scans(dtype):
    """Tokens come in blocks of 64, which are counted below 2^31."""
    for n, fits in (((1 << 31) - 1, False), ((1 << 31) - 63, False), ((1 << 31) - 64, True)):
        need = capi.hla_ssm_workspace_bytes(1, n, 1, 16, 1, 16, dtype)
        # 16 bytes a token, and the ends
        assert (16 * n <= need < 17 * n) if fits else need == 0
        _refused(_ssm(n=n, H=1, dtt=1, ty=dtype, y=P, ws=None), *((capi.HLA_ERR_WORKSPACE, "workspace of") if fits else
                                                                  (UNSUP, "too long")))


@pytest.mark.parametrize("D,K,fits", [((1 << 26) - 16, 3, True), ((1 << 26) - 15, 3, False), (1 << 27, 2, False), (500000000, 4, False),
                                      (50000000, 4, True)])
def test_conv_gradient_widths(D, K, fits):
    """The sums over the tokens take 16 threads a weight or bias, of less than 2^32."""
    assert (capi.hla_conv_backward_workspace_bytes(1, 1, D, K) > 0) == fits
    rc = capi.lib().hla_conv_backward(P, 0, D, P, None, P, 0, D, P, P, None, 1, 1, D, K, 1, BF16, BF16, None, 0, None)
    _refused(rc, *((capi.HLA_ERR_WORKSPACE, "workspace of") if fits else (UNSUP, "too wide")))
    assert _conv(n=1, xt=D, D=D, K=K) == INVALID and "y is NULL" in capi.hla_last_error()


def test_strides_of_size_one_dimensions_are_not_used():
    """One sequence has no distance to the next, one token none to the next:
    whatever stands there is not looked at, odd and negative values included."""
    for kw in (dict(xb=-1), dict(xt=-1, n=1), dict(xb=-3, xt=-5, n=1)):
        _refused(_conv(**kw), INVALID, "y is NULL")
    for kw in (dict(qb=-1), dict(qb=3), dict(qt=-1, kt=3, n=1)):
        _refused(_qk(**kw), INVALID, "k_out is NULL")
    for kw in (dict(xb=3), dict(xb=-1), dict(xt=3, bt=-1, dtt=-1, n=1), dict(dtb=-1)):
        _refused(_scan(**kw), INVALID, "y is NULL")
    _refused(capi.lib().hla_ssm_step(P, P, -1, P, -1, P, P, 3, P, 5, None, None, None, 1, 2, 64, 1, 64, 1, BF16, BF16, None),
             INVALID, "y is NULL")
    _refused(capi.lib().hla_conv_backward(P, -1, -1, P, None, P, -1, -1, None, P, None, 1, 1, 64, 4, 1, BF16, BF16, P, 1 << 30,
                                          None), INVALID, "dx is NULL")
    _refused(capi.lib().hla_ssm_backward(P, -1, 3, P, -1, -1, P, P, 3, 3, P, 3, 3, None, None, P, -1, 3, None, P, P, P, P, None,
                                         None, 1, 1, 2, 64, 1, 64, 1, BF16, BF16, P, 1 << 40, None), INVALID, "dx is NULL")
    # two of them are looked at
    _refused(_conv(B=2, xb=-1), INVALID, "strides")
    _refused(_qk(B=2, qb=3), INVALID, "whole 16-byte")
    _refused(_scan(B=2, xb=3), INVALID, "whole 16-byte")
    _refused(_scan(B=2, xb=1024, dtb=-1), INVALID, "strides")


def _scan(B=1, n=8, xb=0, xt=128, dtb=0, dtt=2, bt=64):
    return capi.lib().hla_ssm_forward(P, xb, xt, P, dtb, dtt, P, P, 0, bt, P, 0, 64, None, None, None, None, B, n, 2, 64, 1, 64,
                                      1, BF16, BF16, P, 1 << 40, None)


@pytest.mark.parametrize("B,H,fits", [(2048, 32, True), ((1 << 24) - 1, 1, True), (1 << 12, 1 << 12, False), (1 << 20, 1 << 20, False)])
def test_heads_of_a_step(B, H, fits):
    """A workgroup a head, 2^32 threads; more than the scan's 65535 heads, which are a grid's second dimension."""
    rc = capi.lib().hla_ssm_step(P, P, H * 16, P, H, P, P, 16, P, 16, None, None, None, B, H, 16, 1, 16, 1, BF16, BF16, None)
    _refused(rc, *((INVALID, "y is NULL") if fits else (UNSUP, "B*H")))
    assert capi.hla_ssm_workspace_bytes(2048, 1, 32, 16, 1, 16, BF16) == 0 and "65535" in capi.hla_last_error()


def test_the_binding_keeps_the_librarys_error_codes(monkeypatch):
    """Sizes whose workspace query refuses them: the error has the entry's code, not one of its own."""
    import torch

    from paper_2510_27258_amd import mixer
    monkeypatch.setattr(mixer, "_on_gpu", lambda t: None)
    monkeypatch.setattr(mixer, "_launch", lambda entry, t, *args: entry(*args, None))

    def z(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)

    def scan(P, dtype=torch.bfloat16):
        return z(1, 4, 2, P, dtype=dtype), z(1, 4, 2), z(2, dtype=torch.float32), z(1, 4, 1, 16, dtype=dtype), z(1, 4, 1, 16,
                                                                                                            dtype=dtype)
    wide, fp32 = scan(24), scan(16, torch.float32)
    for code, text, call in ((UNSUP, "P and N", lambda: mixer.ssm_forward(*wide)),
                             (UNSUP, "P and N", lambda: mixer.ssm_backward(*wide, None, None, wide[0])),
                             (UNSUP, "bf16", lambda: mixer.ssm_backward(*fp32, None, None, fp32[0])),
                             (UNSUP, "K must be", lambda: mixer.conv_backward(z(1, 4, 8), z(8, 5), None, z(1, 4, 8))),
                             (INVALID, "B, n and D", lambda: mixer.conv_backward(z(1, 0, 8), z(8, 4), None, z(1, 0, 8)))):
        with pytest.raises(capi.HLAError) as e:
            call()
        assert e.value.code == code and text in str(e.value), (code, str(e.value))
