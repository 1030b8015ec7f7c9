"""Backward passes through kernels, which have no derivatives of their own."""
from __future__ import annotations

import functools

import torch


class _FirstOnly(torch.autograd.Function):
    """A gradient as it is; asking for its derivative is an error."""

    @staticmethod
    def forward(ctx, g, *anchors):
        return g.view_as(g)

    @staticmethod
    def backward(ctx, dg):
        raise RuntimeError("no second derivatives here: the gradients of these kernels are not recorded")


def anchor(like):
    """One more result of a function, of no size, which it returns and saves: the saved
    one leads back to the function and so to its inputs, and keeps none of them."""
    return like.new_empty(0, dtype=torch.float32)


def first_derivatives_only(backward):
    """A backward pass through kernels, backward(ctx, saved tensors, dZ): where a graph
    of it is asked for (create_graph), its results lead to an error and not to a part
    that is missing.  They hang on the output gradient and on what was saved, as far as
    those require gradients, so that a derivative with respect to any of them finds the
    error.  A function that does not save an input that its gradients depend on (but a
    packed copy, which has no graph) saves an anchor(): through it they hang on all of
    its inputs.  What was saved is asked for once: a checkpoint computes it anew for that."""

    @functools.wraps(backward)
    def wrapped(ctx, dZ, *_):  # an anchor's gradient means nothing
        kept = ctx.saved_tensors
        if not torch.is_grad_enabled():
            return backward(ctx, kept, dZ)
        with torch.no_grad():
            grads = backward(ctx, kept, dZ)
        anchors = [v for v in (dZ, *kept) if v is not None and v.requires_grad]
        anchors = anchors or [dZ.new_empty(0).requires_grad_()]
        return tuple(g if g is None else _FirstOnly.apply(g, *anchors) for g in grads)

    return wrapped
