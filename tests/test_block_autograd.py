"""What automatic differentiation may and may not do with the differentiable
operators of a block, without a GPU: the launches are stubbed, so the values
mean nothing; whether derivatives are taken or refused does."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2510_27258_amd import block

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def stubbed(monkeypatch):
    launched = []

    def launch(entry, t, *args):
        launched.append(entry.__name__)
    monkeypatch.setattr(block, "_launch", launch)
    monkeypatch.setattr(block, "_on_gpu", lambda t: None)
    return launched


def _calls():
    """name: (operator of its learned tensors, those tensors)."""
    z = lambda *s, t=BF16: torch.zeros(*s, dtype=t)  # noqa: E731
    return {
        "gated norm": (lambda y, g, w: block.gated_norm(y, g, w), [z(2, 8, 4, 16), z(2, 8, 4, 16), z(4, 16)]),
        "residual norm": (lambda x, y, w, p, s: torch.cat([o.flatten() for o in block.residual_norm(x, y, w, p, s)]),
                          [z(2, 8, 16, t=F32), z(2, 8, 16), z(16), z(16), z(16)]),
        "recurrence": (lambda *a: block.glr_scan(*a), [z(2, 8, 16), z(2, 8, 16), z(2, 8, 16), z(16, t=F32), z(16, t=F32),
                                                       z(16, t=F32)]),
        "projections": (lambda x, g, u: block.glu(x, g, u), [z(2, 8, 16), z(24, 16), z(24, 16)]),
    }


NAMES = sorted(_calls())


@pytest.mark.parametrize("name", NAMES)
def test_forward_mode_is_refused(name):
    op, args = _calls()[name]
    for i in range(len(args)):
        with fwd.dual_level():
            dual = [fwd.make_dual(a, torch.ones_like(a)) if j == i else a for j, a in enumerate(args)]
            with pytest.raises(NotImplementedError):
                op(*dual)


@pytest.mark.parametrize("name", NAMES)
def test_function_transforms_are_refused(name):
    op, args = _calls()[name]
    with pytest.raises((RuntimeError, NotImplementedError)):
        torch.func.jvp(op, tuple(args), tuple(torch.ones_like(a) for a in args))
    with pytest.raises((RuntimeError, NotImplementedError)):
        torch.func.grad(lambda *a: op(*a).sum())(*args)
    with pytest.raises((RuntimeError, NotImplementedError)):
        torch.vmap(op)(*(a[None] for a in args))


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(name):
    op, args = _calls()[name]
    args = [a.requires_grad_() for a in args]
    grads = torch.autograd.grad(op(*args).sum(), args, create_graph=True)
    for g in grads:
        for a in args:
            with pytest.raises(RuntimeError, match="differentiable once"):
                torch.autograd.grad(g.sum(), a, retain_graph=True)


@pytest.mark.parametrize("name", NAMES)
def test_gradients_have_their_inputs_shapes_and_types(name):
    op, args = _calls()[name]
    for i in range(len(args)):            # one learned input at a time
        one = [a.clone().requires_grad_(j == i) for j, a in enumerate(args)]
        (g,) = torch.autograd.grad(op(*one).sum(), [one[i]])
        assert g.shape == one[i].shape and g.dtype == one[i].dtype


def test_without_gradients_only_the_forward_runs(stubbed):
    for name in NAMES:
        op, args = _calls()[name]
        del stubbed[:]
        op(*args)
        with torch.no_grad():
            op(*(a.requires_grad_() for a in args))
        assert len(stubbed) == 2 and not any("backward" in s for s in stubbed), (name, stubbed)


@pytest.mark.parametrize("which", [0, 1])
def test_one_output_of_the_residual_norm(stubbed, which, monkeypatch):
    """An output that nothing follows has no upstream gradient: none is made up."""
    seen = []
    real = block.residual_norm_backward
    monkeypatch.setattr(block, "residual_norm_backward", lambda *a: (seen.append(a[5:7]), real(*a))[1])
    x, y = torch.zeros(2, 8, 16, requires_grad=True), torch.zeros(2, 8, 16)
    block.residual_norm(x, y)[which].sum().backward()
    assert (seen[0][0] is None, seen[0][1] is None) == (which == 1, which == 0)


def test_the_gradient_of_a_transposed_view_is_laid_out_as_it():
    y = torch.zeros(2, 4, 8, 16).transpose(1, 2).requires_grad_()
    (g,) = torch.autograd.grad(block.gated_norm(y).sum(), y)
    assert g.stride() == y.stride()
    y = torch.zeros(2, 8, 1, 16).expand(2, 8, 4, 16).requires_grad_()       # repeated rows: no layout to copy
    (g,) = torch.autograd.grad(block.gated_norm(y).sum(), y)
    assert g.is_contiguous()
