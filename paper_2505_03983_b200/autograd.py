"""The operators that have gradients, as torch.autograd functions of the current device's handle.

    y, s = add_rmsnorm(x, weight, residual)      y = norm(x + residual) * weight, s = x + residual
    y = gated_mlp(x, w_in, w_out, act)           y = (act(x Wg^T) * (x Wu^T)) w_out^T

They have first derivatives only: a gradient that was made with create_graph=True raises where it is differentiated through one of
these functions.
"""
from __future__ import annotations

import torch

from .operators import default_ops


class _FirstOnly(torch.autograd.Function):
    """Gradients that were computed without a graph, tied to what they depend on by a derivative that raises.
    torch.autograd.function.once_differentiable does so only where a gradient that comes in requires one itself, and so lets the
    derivative of a fixed direction (a divergence) pass for a constant."""

    @staticmethod
    def forward(ctx, n, *tensors):
        return tuple(t.view_as(t) for t in tensors[:n])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("add_rmsnorm and gated_mlp have first derivatives only: differentiating their gradients is not supported")


def _first_only(grads, *depend_on):
    """grads (None among them), as a backward pass returns them."""
    if not torch.is_grad_enabled():  # no create_graph
        return grads
    made = [g for g in grads if g is not None]
    tied = iter(_FirstOnly.apply(len(made), *made, *(t for t in depend_on if t is not None)))
    return tuple(None if g is None else next(tied) for g in grads)


class _AddRmsnorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, s = default_ops().add_rmsnorm(x, weight, residual=residual, eps=eps)
        ctx.save_for_backward(s, weight)
        ctx.set_materialize_grads(False)
        ctx.eps, ctx.has_residual = eps, residual is not None
        return y, s if residual is not None else s.view_as(s)  # without a residual s is x: an output of its own

    @staticmethod
    def backward(ctx, dy, ds):
        s, weight = ctx.saved_tensors
        need_dw = weight is not None and ctx.needs_input_grad[1]
        need_dx = ctx.needs_input_grad[0] or ctx.needs_input_grad[2]
        if dy is None:  # only s was used
            return ds, torch.zeros_like(weight) if need_dw else None, ds if ctx.has_residual else None, None
        dx, dw = default_ops().add_rmsnorm_backward(dy, s, weight, ds=ds if need_dx else None, eps=ctx.eps, need_dweight=need_dw, need_dx=need_dx)
        dx, dw = _first_only((dx, dw), s, weight, dy, ds)
        return dx, dw, dx if ctx.has_residual else None, None


class _GatedMlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_in, w_out, act, keep):
        ctx.act = act
        if not keep:
            return default_ops().gated_mlp(x, w_in, w_out, act=act)
        y, saved = default_ops().gated_mlp_forward(x, w_in, w_out, act=act)
        ctx.save_for_backward(x, w_in, w_out, saved)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w_in, w_out, saved = ctx.saved_tensors
        grads = default_ops().gated_mlp_backward(dy, x, w_in, w_out, saved, act=ctx.act, need=ctx.needs_input_grad[:3])
        return (*_first_only(grads, x, w_in, w_out, dy), None, None)


def add_rmsnorm(x, weight, residual=None, eps=1e-6):
    """AsdOps.add_rmsnorm with gradients in x, weight and residual."""
    return _AddRmsnorm.apply(x, weight, residual, eps)


def gated_mlp(x, w_in, w_out, act="silu"):
    """AsdOps.gated_mlp with gradients in x, w_in and w_out."""
    # in the function itself needs_input_grad would be true of a parameter under no_grad too
    keep = torch.is_grad_enabled() and (x.requires_grad or w_in.requires_grad or w_out.requires_grad)
    return _GatedMlp.apply(x, w_in, w_out, act, keep)
