"""The training operators as differentiable functions.

    from paper_2403_06988_amd import autograd as dva

    x = dva.embed(table, ids, scale)                        # [N][D]
    loss = dva.head_loss(x, weight, targets, allow, states)  # [N]
    loss = dva.distill_loss(logits, teacher_ids, teacher_logits, inv_t, allow, states)
    x, total = dva.rms_norm(hidden, gain, eps, residual)     # [N][D] each
    logits = dva.linear_f8(x, weight)                        # [N][V], products of 8-bit operands

Arguments and results are those of the package's calls of the same names;
gradients reach tables, weights, hidden states and logits.  Each works out its
gradient when the backward pass asks for it, from the inputs (and the head loss's
logarithms of sums): no logits and no probabilities are kept.  ``linear_f8`` keeps its
input and weight in 8 bits only (a byte an element and a scale for 128 of them).  A
gradient of gradients raises.  A program that knows
its rows' weights beforehand calls the ``_backward`` functions itself:
``distill_loss_backward`` gives loss and gradient in one pass over the logits, and
``embed_backward`` with ``accumulate`` adds to a shared table's gradient in place.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

import paper_2403_06988_amd as dv

__all__ = ["embed", "head_loss", "distill_loss", "rms_norm", "linear_f8"]


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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        out, total, rstd = dv.rms_norm(x, weight, eps, residual=residual, want_rstd=True)
        ctx.save_for_backward(x if total is None else total, weight, rstd)
        ctx.has_residual = residual is not None
        ctx.set_materialize_grads(False)
        return (out, total) if ctx.has_residual else out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out, grad_total=None):
        total, weight, rstd = ctx.saved_tensors
        want_x, want_weight = any(ctx.needs_input_grad[:2]), ctx.needs_input_grad[2]
        if grad_out is None:
            grad_x, grad_weight = grad_total, None
        else:
            grad_x, grad_weight = dv.rms_norm_backward(
                grad_out.contiguous(), total, weight, rstd,
                grad_total=None if grad_total is None else grad_total.contiguous(), want_x=want_x, want_weight=want_weight)
        return grad_x, grad_x if ctx.has_residual else None, grad_weight, None


class _LinearF8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, exact):
        want_x, want_weight = ctx.needs_input_grad[:2]
        q, scales, t_q, t_scales = dv.quantize_f8(x, want_columns=want_weight)
        w_q, w_scales, wt_q, wt_scales = dv.quantize_f8(weight, tile=dv.SCALE_BLOCK, want_columns=want_x)
        ctx.save_for_backward(t_q, t_scales, wt_q, wt_scales)
        ctx.weight_shape, ctx.weight_dtype, ctx.exact = weight.shape, weight.dtype, exact
        return dv.product_f8(q, scales, w_q, w_scales, tile=dv.SCALE_BLOCK, dtype=x.dtype, exact=exact)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        t_q, t_scales, wt_q, wt_scales = ctx.saved_tensors
        want_x, want_weight = ctx.needs_input_grad[:2]
        g_q, g_scales, gt_q, gt_scales = dv.quantize_f8(grad_out.contiguous(), want_rows=want_x, want_columns=want_weight)
        grad_x = grad_weight = None
        if want_x:
            grad_x = dv.product_f8(g_q, g_scales, wt_q, wt_scales, tile=dv.SCALE_BLOCK, dtype=grad_out.dtype, exact=ctx.exact)
        if want_weight and grad_out.shape[0] == 0:  # a sum of nothing
            grad_weight = grad_out.new_zeros(ctx.weight_shape, dtype=ctx.weight_dtype)
        elif want_weight:
            grad_weight = dv.product_f8(gt_q, gt_scales, t_q, t_scales, tile=1, dtype=ctx.weight_dtype, exact=ctx.exact)
        return grad_x, grad_weight, None


def embed(weight, ids, scale=1.0):
    """``dv.embed``; the gradient reaches ``weight``."""
    return _Embed.apply(weight, ids, scale)


def head_loss(x, weight, targets, allow=None, states=None):
    """The loss of ``dv.head_loss`` [N]; gradients reach ``x`` and ``weight``."""
    return _HeadLoss.apply(x, weight, targets, allow, states)


def distill_loss(logits, teacher_ids, teacher_logits, inv_temperature=1.0, allow=None, states=None):
    """``dv.distill_loss`` [N]; the gradient reaches ``logits``."""
    return _DistillLoss.apply(logits, teacher_ids, teacher_logits, inv_temperature, allow, states)


def rms_norm(x, weight, eps=1e-6, residual=None):
    """``dv.rms_norm``: its result, or with a residual (result, x + residual);
    gradients reach ``x``, ``weight`` and ``residual``."""
    return _RmsNorm.apply(x, residual, weight, eps)


def linear_f8(x, weight, exact=False):
    """x weight^T [N][V] of x [N][D] and weight [V][D], all three products (this
    and both gradients') of 8-bit operands: x and the gradient with a scale for
    every 128 elements along the products' sums, the weight for every 128 x 128.
    Sums are in fp32, the result and x's gradient in x's type, the weight's in the
    weight's, which may be another.  ``exact``: bfloat16 results with the sums of
    float32 ones, as ``dv.product_f8``."""
    if x.dim() != 2 or weight.dim() != 2 or weight.shape[1] != x.shape[1]:  # (padded to whole blocks both might fit)
        raise ValueError(f"x must be [N][D] and weight must be [V][D], got {list(x.shape)} and {list(weight.shape)}")
    return _LinearF8.apply(x, weight, exact)
