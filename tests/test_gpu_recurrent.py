"""The operators of a block together, as examples/recurrent.py uses them: a
training step that reaches every parameter with the gradients of the same model
in fp64, and a prompt with single tokens that give the whole sequence's logits.

The model's activations are bf16: a chain of some twenty roundings of 2^-8, each
of its own sign, so a gradient is held to 2^-4 of its 2-norm, and served logits,
which go through the same roundings in another order, to 2^-4 of the largest."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent.py")


@pytest.fixture(scope="module")
def recurrent():
    spec = importlib.util.spec_from_file_location("recurrent", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _model(recurrent):
    torch.manual_seed(0)
    return recurrent.Recurrent().cuda().bfloat16()


def _norm(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _plain(model, p, ids):
    """The model's forward in fp64 with parameters p, from the formulas."""
    x = stream = p["embed.weight"][ids]
    u = _norm(x, p["first"])
    for i in range(len(model.mixers)):
        m = {k[len(f"mixers.{i}."):]: v for k, v in p.items() if k.startswith(f"mixers.{i}.")}
        inner, n = model.mixers[i].inner, ids.shape[1]
        c, f, g, z = (u @ m["proj.weight"].T).split(inner, -1)
        past = F.pad(c, (0, 0, 3, 0))
        c = F.silu(sum(past[:, j:j + n] * m["conv"][:, j] for j in range(4)))
        la = -8 * F.softplus(m["decay"]) * torch.sigmoid(f + m["f_bias"])
        b = torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(g + m["g_bias"]) * c
        h, hs = torch.zeros_like(b[:, 0]), []
        for t in range(n):
            h = la[:, t].exp() * h + b[:, t]
            hs.append(h)
        h = torch.stack(hs, 1)
        v = (h * F.silu(z)).unflatten(-1, (inner // 64, 64))
        u = _norm(v, m["norm"]).flatten(2) @ m["out.weight"].T
        for k in (2 * i, 2 * i + 1):
            if k % 2:
                gate, up = p[f"mlps.{i}.gate"], p[f"mlps.{i}.up"]
                u = (F.silu(u @ gate.T) * (u @ up.T)) @ p[f"mlps.{i}.down.weight"].T
            stream = stream + p[f"scale.{k}"] * _norm(u, p[f"after.{k}"])
            u = _norm(stream, p[f"before.{k}"])
    return u @ p["head.weight"].T


def test_training_gradients(recurrent):
    model = _model(recurrent)
    ids = recurrent.sequences(3, 41, 17, torch.Generator("cuda").manual_seed(5))
    target = ids[:, 1:].flatten()
    F.cross_entropy(model(ids[:, :-1]).flatten(0, 1), target).backward()
    p = {k: v.detach().double().requires_grad_() for k, v in model.named_parameters()}
    F.cross_entropy(_plain(model, p, ids[:, :-1]).flatten(0, 1), target).backward()
    for name, v in model.named_parameters():
        ref = p[name].grad
        assert ref.norm() > 0 and (v.grad.double() - ref).norm() <= 2 ** -4 * ref.norm(), name


def test_training_runs(recurrent):
    model = _model(recurrent)
    losses = recurrent.train(model, 3, B=4, n=130, say=None)
    assert all(torch.isfinite(torch.tensor(losses)))
    assert all(torch.isfinite(p.grad).all() and p.grad.abs().max() > 0 for p in model.parameters())


@pytest.mark.parametrize("n", [1, 65, 130])
def test_prompt_and_steps_give_the_whole_sequences_logits(recurrent, n):
    model = _model(recurrent)
    ids = recurrent.sequences(3, n, 17, torch.Generator("cuda").manual_seed(n))
    out, logits = recurrent.generate(model, ids, 20)
    with torch.no_grad():
        whole = model(out[:, :-1])[:, -20:]
    assert (logits - whole).abs().max() <= 2 ** -4 * whole.abs().max()
