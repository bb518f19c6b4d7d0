"""The training operators as differentiable functions.

    from paper_2403_06988_amd import autograd as dva

    x = dva.embed(table, ids, scale)                        # [N][D]
    loss = dva.head_loss(x, weight, targets, allow, states)  # [N]
    loss = dva.distill_loss(logits, teacher_ids, teacher_logits, inv_t, allow, states)

Arguments and results are those of the package's calls of the same names;
gradients reach tables, weights, hidden states and logits.  Each works out its
gradient when the backward pass asks for it, from the inputs (and the head loss's
logarithms of sums): no logits and no probabilities are kept.  A gradient of
gradients raises.  A program that knows
its rows' weights beforehand calls the ``_backward`` functions itself:
``distill_loss_backward`` gives loss and gradient in one pass over the logits, and
``embed_backward`` with ``accumulate`` adds to a shared table's gradient in place.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

import paper_2403_06988_amd as dv

__all__ = ["embed", "head_loss", "distill_loss"]


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, ids, scale):
        ctx.save_for_backward(ids)
        ctx.num_tokens, ctx.scale = weight.shape[0], scale
        return dv.embed(weight, ids, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        (ids,) = ctx.saved_tensors
        return dv.embed_backward(grad_out.contiguous(), ids, ctx.num_tokens, ctx.scale), None, None


class _HeadLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets, allow, states):
        loss, lse = dv.head_loss(x, weight, targets, allow, states)
        ctx.save_for_backward(x, weight, targets, allow, states, lse)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss):
        x, weight, targets, allow, states, lse = ctx.saved_tensors
        want_x, want_weight = ctx.needs_input_grad[:2]
        grad_x, grad_weight = dv.head_loss_backward(x, weight, targets, lse, grad_loss.contiguous(), allow, states,
                                                    want_x=want_x, want_weight=want_weight)
        return grad_x, grad_weight, None, None, None


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, inv_temperature, allow, states):
        ctx.save_for_backward(logits, teacher_ids, teacher_logits, allow, states)
        ctx.inv_temperature = inv_temperature
        return dv.distill_loss(logits, teacher_ids, teacher_logits, inv_temperature, allow, states)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss):
        logits, teacher_ids, teacher_logits, allow, states = ctx.saved_tensors
        _, grad = dv.distill_loss_backward(logits, teacher_ids, teacher_logits, grad_loss.contiguous(),
                                           ctx.inv_temperature, allow, states)
        return grad, None, None, None, None, None


def embed(weight, ids, scale=1.0):
    """``dv.embed``; the gradient reaches ``weight``."""
    return _Embed.apply(weight, ids, scale)


def head_loss(x, weight, targets, allow=None, states=None):
    """The loss of ``dv.head_loss`` [N]; gradients reach ``x`` and ``weight``."""
    return _HeadLoss.apply(x, weight, targets, allow, states)


def distill_loss(logits, teacher_ids, teacher_logits, inv_temperature=1.0, allow=None, states=None):
    """``dv.distill_loss`` [N]; the gradient reaches ``logits``."""
    return _DistillLoss.apply(logits, teacher_ids, teacher_logits, inv_temperature, allow, states)
