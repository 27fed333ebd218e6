"""Infinite gate inputs of the recurrence shut and open their gates as those of
+-200 do, whose sigmoids are 0 and 1 in fp32: the same bits, all finite."""
import pytest
import torch

import paper_2510_27258_amd as hla
from tests.test_gpu_block import BF16, FP32, _glr_case, _say
from tests.test_gpu_block_edges import _same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", [(2, 300, 12), (1, 5000, 8), (3, 40, 7)])
def test_infinite_gates(size, dtype):
    x, f, g, decay, fb, gb, dy, state = _glr_case(*size, dtype, True, 91)
    got = []
    for far in (200.0, float("inf")):
        _say(f"infinite gates {size} {dtype} {far}")
        f2, g2, st = f.contiguous(), g.contiguous(), state.clone()
        f2[:, 3::5, 0::4], f2[:, 1::3, 1::4] = -far, far
        g2[:, 2::7, 0::3], g2[:, 4::5, 2::3] = far, -far
        outs = [hla.glr_prefill(st, x, f2, g2, decay, fb, gb), st.clone()]
        outs += [hla.glr_step(st, x[:, 3], f2[:, 3], g2[:, 3], decay, fb, gb), st]
        got.append(outs + list(hla.glr_backward(x, f2, g2, decay, fb, gb, dy)))
    for a, b in zip(*got):
        assert torch.isfinite(b.float()).all() and _same(a, b)
