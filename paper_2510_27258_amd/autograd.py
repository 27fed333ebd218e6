"""What the library's autograd functions share."""
import functools

import torch


class _Once(torch.autograd.Function):
    """The first `count` tensors as they are, part of the graph of all that
    follow them, which cannot be differentiated."""

    @staticmethod
    def forward(ctx, count, *tensors):
        return tensors[:count]

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of this operator cannot be differentiated: it is differentiable once")


def once(backward):
    """A function's backward without second derivatives.  Its kernels leave no
    graph, so with create_graph=True its gradients would be constants: here
    they depend on the saved tensors and on the upstream gradients, and raise
    where they are differentiated.  (torch's own once_differentiable raises for
    the upstream gradients only, and a gradient is a function of the inputs
    also where its upstream gradient is a constant.)"""
    @functools.wraps(backward)
    def wrapped(ctx, *upstream):
        if not torch.is_grad_enabled():
            return backward(ctx, *upstream)
        with torch.no_grad():
            grads = backward(ctx, *upstream)
        given = [g for g in grads if g is not None]
        kept = iter(_Once.apply(len(given), *given, *ctx.saved_tensors, *upstream))
        return tuple(None if g is None else next(kept) for g in grads)
    return wrapped
