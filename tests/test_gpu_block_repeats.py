"""The operators of a block at the sizes of a training batch, where a workgroup
takes several tiles one behind the other, sequences are cut and long sums are
joined from parts: the same inputs give the same bits, whatever ran between."""
import pytest
import torch

import paper_2510_27258_amd as hla
from tests.test_gpu_block import BF16, _say
from tests.test_gpu_block_edges import _all, _same

pytestmark = pytest.mark.gpu


def _projections(draw, act):
    x, dh = draw(4, 4096, 1024), draw(4, 4096, 4096)
    wg, wu = draw(4096, 1024) / 32, draw(4096, 1024) / 32
    return lambda: (hla.glu_forward(x, wg, wu, act), *hla.glu_backward(x, wg, wu, dh, act))


def _recurrence(draw, B, n, D):
    x, f, g, dy = (draw(B, n, D) for _ in range(4))
    decay, bias = torch.linspace(-6, -3, D, device="cuda"), torch.linspace(-1, 1, D, device="cuda")
    return lambda: (hla.glr_forward(x, f, g, decay, bias, bias), *hla.glr_backward(x, f, g, decay, bias, bias, dy))


def _norms(draw, n, D):
    x, y, go, gr = (draw(2, n, D) for _ in range(4))
    ws = [draw(D) for _ in range(3)]
    heads = [t.unflatten(-1, (-1, D // 16)) for t in (x, y, go)]
    w = draw(16, D // 16)
    return lambda: (*hla.residual_norm_forward(x, y, *ws), *hla.residual_norm_backward(x, y, *ws, go, gr),
                    *hla.gated_norm_backward(heads[0], heads[1], w, heads[2]))


CASES = {
    "projections, SiLU": lambda draw: _projections(draw, "silu"),
    "projections, GELU": lambda draw: _projections(draw, "gelu"),
    "recurrence": lambda draw: _recurrence(draw, 4, 4096, 2048),
    "recurrence in segments": lambda draw: _recurrence(draw, 1, 16384, 1024),
    "recurrence of single channels": lambda draw: _recurrence(draw, 2, 5000, 333),
    "norms": lambda draw: _norms(draw, 4096, 1024),
    "norms of wide rows": lambda draw: _norms(draw, 300, 16384),
}


@pytest.mark.parametrize("name", list(CASES))
def test_the_same_bits(name):
    gen = torch.Generator("cuda").manual_seed(81)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF16)  # noqa: E731
    one, other = CASES[name](draw), CASES[name](draw)
    _say(f"repeats of {name}")
    first, between = _all(one()), _all(other())
    for k in range(4):
        for u, v in zip(between, _all(other())):
            assert _same(u, v), (name, k)
        for u, v in zip(first, _all(one())):
            assert _same(u, v), (name, k)
