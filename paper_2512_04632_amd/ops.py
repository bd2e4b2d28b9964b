"""The library's operators with automatic differentiation.

Thin front ends of the entry points in ``_lib`` for training: layer norm and
root-mean-square norm, the routing of rows to experts, rows on their way to the
experts' order and back, products of ragged groups of rows with one matrix per
expert, the log probabilities of given tokens, and the clipped policy loss with
a KL term.  The arithmetic runs in the library's kernels;
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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        ctx.set_materialize_grads(False)
        y, s, rstd = _lib.rms_norm(x, weight, residual, eps)
        ctx.save_for_backward(s, weight, rstd)
        ctx.added = residual is not None
        return (y, s) if ctx.added else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds=None):
        s, weight, rstd = ctx.saved_tensors
        dweight = None
        if dy is not None:
            ds, dweight = _lib.rms_norm_backward(dy, s, rstd, weight, ds, param_grads=ctx.needs_input_grad[1])
        return ds, dweight, ds if ctx.added else None, None


def rms_norm(x, weight=None, residual=None, eps: float = 1e-5):
    """Root-mean-square norm over the last dimension (bf16 or fp32 x; fp32 weight, or None).

    With a residual of x's shape and type, (y, s): s = x + residual is normalised and goes on as
    the residual stream; without one y alone."""
    return _RmsNorm.apply(x, weight, residual, eps)


class _ExpertRoute(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top, active, renormalize, scale):
        ctx.set_materialize_grads(False)
        chosen, weights, slots, ends, balance = _lib.expert_route(logits, top, active, renormalize, scale)
        ctx.save_for_backward(logits, chosen, ends)
        ctx.how = renormalize, scale
        ctx.mark_non_differentiable(chosen, slots, ends)
        return weights, balance, chosen, slots, ends

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, dbalance, *_):
        logits, chosen, ends = ctx.saved_tensors
        if dweights is None and dbalance is None:
            return (None,) * 5
        return (_lib.expert_route_backward(logits, chosen, ends, dweights, dbalance, *ctx.how),) + (None,) * 4


def expert_route(logits, top: int, active=None, renormalize: bool = True, scale: float = 1.0):
    """(weights, balance, chosen, slots, ends): the `top` experts of each row of scores, see
    _lib.expert_route.  The weights and the balance loss are differentiated by the logits (the
    choices, and with them the experts' shares of the rows, are taken as given)."""
    return _ExpertRoute.apply(logits, top, active, renormalize, scale)


class _ExpertGather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, slots, ends):
        ctx.save_for_backward(slots, ends)
        return _lib.expert_gather(x, slots, ends)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        slots, ends = ctx.saved_tensors
        return _lib.expert_combine(dout, slots, ends=ends), None, None


def expert_gather(x, slots, ends=None):
    """The rows of x in the experts' order, as expert_linear takes them: out[slots[i, j]] = x[i] for
    expert_route's slots and ends; zeros from ends[-1] on.  Without ends, zeros in every row that no slot
    names (another pass): so for slots with choices taken out, as with ends every row below ends[-1]
    has to be in a slot."""
    return _ExpertGather.apply(x, slots, ends)


class _ExpertCombine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, slots, weights, residual, ends):
        ctx.save_for_backward(y, slots, weights, ends)
        return _lib.expert_combine(y, slots, weights, residual, ends)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        y, slots, weights, ends = ctx.saved_tensors
        dy = dweights = None
        if ctx.needs_input_grad[0] or ctx.needs_input_grad[2]:
            dy, dweights = _lib.expert_combine_backward(dout, y, slots, ends, weights,
                                                        weight_grads=ctx.needs_input_grad[2])
        return (dy if ctx.needs_input_grad[0] else None, None, dweights,
                dout if ctx.needs_input_grad[3] else None, None)


def expert_combine(y, slots, weights=None, residual=None, ends=None):
    """residual[i] + sum over j of weights[i, j] y[slots[i, j]]: the experts' results back in the rows'
    order.  ends (expert_route's) says which rows of y are filled: the others have no part in it and a
    gradient of zero, and every one that is has to be in a slot.  Without it rows of y in no slot
    have a gradient of zero (another pass).  For gradients no two slots may be the same."""
    return _ExpertCombine.apply(y, slots, weights, residual, ends)


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


class _TokenLogp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top, temperature):
        ctx.set_materialize_grads(False)
        logp, entropy, stats, top_logp, top_ids = _lib.token_logp(logits, targets, top, temperature)
        ctx.save_for_backward(logits, targets, stats, entropy)
        ctx.temperature = temperature
        if top_ids is None:
            return logp, entropy
        ctx.mark_non_differentiable(top_logp, top_ids)
        return logp, entropy, top_logp, top_ids

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dentropy, *_):
        logits, targets, stats, entropy = ctx.saved_tensors
        if dlogp is None and dentropy is None:
            return (None,) * 4
        grad = _lib.token_logp_backward(logits, targets, stats, entropy, dlogp, dentropy, ctx.temperature)
        return (grad,) + (None,) * 3


def token_logp(logits, targets, top: int = 0, temperature: float = 1.0):
    """(logp, entropy) of int64 targets at the temperature, both differentiated by the logits; with `top`
    also (top_logp, top_ids) of the most likely tokens, which are not.  See _lib.token_logp."""
    return _TokenLogp.apply(logits, targets, top, temperature)
