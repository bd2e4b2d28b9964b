"""The library's operators with automatic differentiation.

Thin front ends of the entry points in ``_lib`` for training: layer norm,
products of ragged groups of rows with one matrix per expert, and the clipped
policy loss with a KL term.  The arithmetic runs in the library's kernels;
this module keeps what a backward pass reads and, where expert matrices are of
another type than the rows, has torch round them.  The gradients of expert
matrices come out stacked, as ``optim.TurboMuon`` takes them.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import _lib


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = _lib.layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        wanted = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dweight, dbias = _lib.layer_norm_backward(dy, x, mean, rstd, weight, param_grads=wanted)
        return (dx, dweight if ctx.needs_input_grad[1] else None, dbias if ctx.needs_input_grad[2] else None, None)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm over the last dimension (bf16 or fp32 x; fp32 weight and bias, or None)."""
    return _LayerNorm.apply(x, weight, bias, eps)


class _ExpertLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, ends):
        wx = w.to(x.dtype)
        ctx.save_for_backward(x, wx, ends)
        ctx.w_dtype = w.dtype
        return _lib.expert_matmul(x, wx, ends)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, wx, ends = ctx.saved_tensors
        dx = _lib.expert_matmul(dy, wx, ends, transposed=True) if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            # rows' own type or fp32 come from the kernel, any other is its fp32 result rounded
            direct = ctx.w_dtype if ctx.w_dtype is x.dtype else torch.float32
            dw = _lib.expert_wgrad(x, dy, ends, dtype=direct).to(ctx.w_dtype)
        return dx, dw, None


def expert_linear(x, w, ends):
    """x[i] @ w[e] for the rows of each expert e: x is (rows, k), rows sorted by expert, w is
    (experts, k, n), ends an int32 device vector with the number of rows up to each expert's last.

    w may be fp32 where x is bf16 (the parameters that the optimizer keeps): torch rounds it to
    bf16 for the products, a copy that is kept for the backward pass, and its gradient comes out
    in fp32.  Any other type of w is taken as x's in the same way, its gradient in its own.
    """
    return _ExpertLinear.apply(x, w, ends)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl, temperature):
        loss, logp, lse, slope = _lib.policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low,
                                                  clip_high, kl, temperature)
        ctx.save_for_backward(logits, targets, lse, slope)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(logp)
        return loss, logp

    @staticmethod
    @once_differentiable
    def backward(ctx, grad, _):
        logits, targets, lse, slope = ctx.saved_tensors
        dlogits = _lib.policy_loss_backward(logits, targets, lse, slope, grad, ctx.temperature)
        return (dlogits,) + (None,) * 9


def policy_loss(logits, targets, old_logp, advantages, weights, ref_logp=None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl: float = 0.0, temperature: float = 1.0):
    """(loss, logp) of the clipped policy loss (see _lib.policy_loss); only the logits are
    differentiated, logp is what the next step keeps as old_logp.

    The gradient takes its probabilities from the row's lse in fp32 and carries its rounding, 2^-24
    of it; for logits of large size use _lib.policy_loss_with_grad, which does not."""
    return _PolicyLoss.apply(logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl,
                             temperature)
