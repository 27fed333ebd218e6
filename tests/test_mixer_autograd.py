"""What automatic differentiation may and may not do with the differentiable
operators, without a GPU: the launches are stubbed, so the values mean nothing;
whether derivatives are taken or refused does."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2510_27258_amd import capi, mixer

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def stubbed(monkeypatch):
    launched = []

    def launch(entry, t, *args):
        launched.append(entry.__name__)
    monkeypatch.setattr(mixer, "_launch", launch)
    monkeypatch.setattr(mixer, "_on_gpu", lambda t: None)
    return launched


def _calls(dtype=BF16):
    """name: (operator of its learned tensors, those tensors)."""
    z = lambda *s, t=dtype: torch.zeros(*s, dtype=t)  # noqa: E731
    f = torch.float32
    return {
        "conv": (lambda x, w, b: mixer.short_conv(x, w, b), [z(2, 8, 16), z(16, 4), z(16)]),
        "qk": (lambda *a: torch.cat([o.flatten() for o in mixer.qk_norm_rope(*a)]),
               [z(2, 8, 4, 64), z(2, 8, 2, 64), z(64), z(64)]),
        "scan": (lambda *a: mixer.ssm_scan(*a),
                 [z(2, 8, 4, 16), z(2, 8, 4), z(4, t=f), z(2, 8, 2, 16), z(2, 8, 2, 16), z(4, t=f), z(4, t=f)]),
    }


NAMES = sorted(_calls())


@pytest.mark.parametrize("name", NAMES)
def test_forward_mode_is_refused(name):
    """No operator has a forward-mode formula: a dual input raises, whichever
    it is, and never loses its tangent silently."""
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
def test_no_graph_without_a_learned_input(name, stubbed):
    op, args = _calls()[name]
    assert not op(*args).requires_grad and len(stubbed) == 1
    args[0].requires_grad_()
    assert op(*args).requires_grad
    with torch.no_grad():
        assert not op(*args).requires_grad


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(name):
    """A gradient taken with a graph cannot be differentiated again: a penalty
    on it raises, also beside a term that can."""
    op, args = _calls()[name]
    for i in range(len(args)):
        leaves = [a.clone().requires_grad_(j == i) for j, a in enumerate(args)]
        out = op(*leaves)
        grad, = torch.autograd.grad(out.float().sum(), leaves[i], create_graph=True)
        assert grad.shape == args[i].shape
        with pytest.raises(RuntimeError, match="differentiable once"):
            (grad.float().square().sum() + leaves[i].float().square().sum()).backward()


def test_second_derivatives_of_the_attention_are_refused(monkeypatch):
    from paper_2510_27258_amd import hla
    monkeypatch.setattr(hla, "forward", lambda q, k, v, chunk: torch.zeros(v.shape))
    monkeypatch.setattr(hla, "_backward", lambda q, k, v, g, chunk, ws, dtype: tuple(torch.zeros_like(t) for t in (q, k, v)))
    args = [torch.zeros(1, 2, 8, 64, dtype=BF16) for _ in range(3)]
    for i in range(3):
        leaves = [a.clone().requires_grad_(j == i) for j, a in enumerate(args)]
        grad, = torch.autograd.grad(hla.hla2_attention(*leaves).sum(), leaves[i], create_graph=True)
        with pytest.raises(RuntimeError, match="differentiable once"):
            (grad.float().square().sum() + leaves[i].float().square().sum()).backward()


def test_fp32_scan_to_be_trained_is_refused_before_its_forward(stubbed):
    """The scan's gradients cover bf16: fp32 inputs that need them raise in
    the forward, not after it."""
    op, args = _calls(torch.float32)["scan"]
    for i in range(len(args)):
        leaves = [a.clone().requires_grad_(j == i) for j, a in enumerate(args)]
        with pytest.raises(capi.HLAError, match="bf16") as e:
            op(*leaves)
        assert e.value.code == capi.HLA_ERR_UNSUPPORTED and not stubbed
    with torch.no_grad():
        op(*leaves)
    assert len(stubbed) == 1
