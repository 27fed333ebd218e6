"""The operators together, as examples/hybrid.py uses them: a training step
that learns, and a prompt with single tokens that give the whole sequence's
logits.

The served logits go through the same bf16 roundings as the whole forward's in
another order (a state instead of a tile's scores); two layers, a head and
their norms leave a few roundings of 2^-8 of the largest logit: 2^-4 is the bar."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid.py")


@pytest.fixture(scope="module")
def hybrid():
    spec = importlib.util.spec_from_file_location("hybrid", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _model(hybrid):
    torch.manual_seed(0)
    return hybrid.Hybrid().cuda().bfloat16()


def test_training_learns_and_reaches_every_parameter(hybrid):
    model = _model(hybrid)
    losses = hybrid.train(model, 40, B=8, n=256, say=None)
    assert all(torch.isfinite(p.grad).all() and p.grad.abs().max() > 0 for p in model.parameters())
    # a model that has learned nothing is at log 17 = 2.83
    assert losses[-1] < 2.0, losses


@pytest.mark.parametrize("n", [1, 65, 130])
def test_prompt_and_steps_give_the_whole_sequences_logits(hybrid, n):
    model = _model(hybrid)
    ids = hybrid.sequences(3, n, 17, torch.Generator("cuda").manual_seed(n))
    out, logits = hybrid.generate(model, ids, 20)
    with torch.no_grad():
        whole = model(out[:, :-1])[:, -20:]
    assert (logits - whole).abs().max() <= 2 ** -4 * whole.abs().max()
