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
