"""The router under torch's automatic differentiation: `route` and `route_backward` as one differentiable call.

    gate, balance, z, r = balanced_route(logits, top_k, fam_off, score="softmax")
    loss = task_loss(gate, r["trace"]) + 0.01 * balance.mean() + 0.001 * z.mean()
    loss.backward()                                      # logits.grad through tacg_route_backward

The selection and the counts are constants of the gradient, as usual for these losses.  There is no second derivative: asking for one
raises.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import _fam_off, route, route_backward


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_k, fam_off, score, bias, renorm, scale, kept):
        r = route(logits, top_k, fam_off, score=score, bias=bias, renorm=renorm, scale=scale, balance=True)
        kept.update(r)
        ctx.save_for_backward(logits, r["trace"], r["norm"], r["D"], r["tokens"])
        ctx.how = (fam_off, score, renorm, scale)
        ctx.set_materialize_grads(False)  # an output without a gradient is left out, not read as zeros
        z = r.get("z")
        return r["gate"], r["balance"], torch.zeros_like(r["balance"]) if z is None else z

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_gate, grad_balance, grad_z):
        logits, trace, norm, D, tokens = ctx.saved_tensors
        fam_off, score, renorm, scale = ctx.how
        whole = lambda g: None if g is None else g.contiguous()  # noqa: E731
        grad = route_backward(logits, trace, norm, fam_off, D=D, tokens=tokens, grad_gate=whole(grad_gate),
                              grad_balance=whole(grad_balance), grad_z=whole(grad_z) if score == "softmax" else None,
                              score=score, renorm=renorm, scale=scale)
        return grad, None, None, None, None, None, None, None


def balanced_route(logits: torch.Tensor, top_k: int, fam_off=None, score: str = "softmax",
                   bias: Optional[torch.Tensor] = None, renorm: bool = False, scale: float = 1.0):
    """(gate [L][N][k], balance [F][L], z [F][L], the dict of `route`): gate, balance and z are differentiable with respect to the
    logits.  z is 0 for sigmoid scores, which have none."""
    kept: dict = {}
    if fam_off is not None:
        fam_off = _fam_off(fam_off).tolist()  # a copy: the backward pass takes the same families, whatever becomes of the caller's
    gate, balance, z = _Route.apply(logits, top_k, fam_off, score, bias, renorm, scale, kept)
    return gate, balance, z, kept
