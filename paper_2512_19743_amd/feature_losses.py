"""PyTorch autograd wrappers of the losses on features and on routed experts (computed in libapml)."""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import _lib


def _upstream(grad_loss: torch.Tensor) -> torch.Tensor:
    return grad_loss if grad_loss.dtype == torch.float32 and grad_loss.is_contiguous() else \
        grad_loss.to(torch.float32).contiguous()


def _linear_ce_grads(ctx, grad_loss):
    x, w, target, state = ctx.saved_tensors
    want_x, want_w = ctx.needs_input_grad[:2]
    gx, gw = _lib._linear_ce_backward(ctx.desc, state, x, w, target, _upstream(grad_loss), want_x, want_w)
    return gx, gw, None, None


class LinearCEFunction(torch.autograd.Function):
    """Softmax cross entropy against classes; the logits are computed again in backward, never kept."""

    @staticmethod
    def forward(ctx, x, w, target, desc):
        need = ctx.needs_input_grad
        loss, state = _lib._linear_ce_forward(desc, x, w, target, need[0] or need[1])
        ctx.desc = desc
        ctx.save_for_backward(x, w, target, state)
        return loss

    @staticmethod
    def backward(ctx, grad_loss):
        if torch.is_grad_enabled():  # create_graph: a second derivative is refused, where one is asked for
            return once_differentiable(_linear_ce_grads)(ctx, grad_loss)
        return _linear_ce_grads(ctx, grad_loss)


def linear_ce_loss(x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, *, scale: float = 1.0,
                   z_weight: float = 0.0, ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """Softmax cross entropy of the rows of x against the classes w, without storing the logits
    scale * x @ w.T; float32, with gradients for x and w in their own type.

    x (..., dim) and w (classes, dim): one set of classes, a code book or a vocabulary. x (B, N, dim) and
    w (B, M, dim): each sample with its own, as when the descriptors of one cloud's points are matched to
    those of the other's (scale, a number: 1 / temperature; a learned one is multiplied into x).
    float32, bfloat16 or float16 GPU tensors, x and w of the same type: autocast does not reach this call, so
    bfloat16 features need a bfloat16 copy of a float32 head. In 16 bits the gradient of the logits is rounded to
    that type, as it would be between two layers, before it is multiplied by w and x.
    target: the rows' classes, int64 or int32, of x's leading shape; ignore_index: a row that adds nothing.
    z_weight: weight of the squared log-sum-exp that is added per row.
    reduction: 'none' (target's shape), 'sum', or 'mean' over the rows that are not ignored.
    """
    x, w, target = x.contiguous(), w.contiguous(), target.contiguous()
    desc = _lib._linear_ce_desc(x, w, target, scale, z_weight, ignore_index, reduction)
    return LinearCEFunction.apply(x, w, target, desc)


def _balance_grads(ctx, grad_loss, _):
    logits, valid, state = ctx.saved_tensors
    grad = _lib._balance_backward(ctx.desc, state, logits, valid, _upstream(grad_loss))
    return grad, None, None, None, None


class BalanceFunction(torch.autograd.Function):
    """Balance loss of routed experts and the tokens per expert; the softmax is computed again in backward."""

    @staticmethod
    def forward(ctx, logits, experts, counts, valid, desc):
        loss, got, state = _lib._balance_forward(desc, logits, experts, counts, valid, ctx.needs_input_grad[0])
        ctx.desc = desc
        ctx.save_for_backward(logits, valid, state)
        if counts is not None:  # an input is no output
            got = logits.new_empty(0, dtype=torch.int64)
        ctx.mark_non_differentiable(got)
        return loss, got

    @staticmethod
    def backward(ctx, grad_loss, grad_counts):
        if torch.is_grad_enabled():  # create_graph: a second derivative is refused, where one is asked for
            return once_differentiable(_balance_grads)(ctx, grad_loss, grad_counts)
        return _balance_grads(ctx, grad_loss, grad_counts)


def balance_loss(logits: torch.Tensor, experts: Optional[torch.Tensor] = None, *, counts: Optional[torch.Tensor] = None,
                 valid: Optional[torch.Tensor] = None, z_weight: float = 0.0, reduction: str = "mean"
                 ) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss, counts): E sum_e f_e P_e per sample, with f_e the share of expert e in the chosen experts and
    P_e the mean of its softmax probability over the valid tokens, plus z_weight times the mean squared
    log-sum-exp; and the tokens per expert, int64.

    logits (B, tokens, experts), a loss per sample, or (tokens, experts), one sample; float32, bfloat16 or
    float16 GPU tensors, up to 1024 experts. experts (..., chosen): the experts that each token goes to, int64 or int32, -1 for
    a dropped slot. counts instead: the tokens per expert, (B, experts) or (experts,), for instance the sum
    of every rank's expert_counts. valid: bool, the tokens' shape, False for padding.
    The gradient flows into logits through the probabilities, not through the counts.
    reduction: 'none' (per sample), 'sum' or 'mean' over the samples.
    """
    logits = logits.contiguous()
    experts, counts, valid = (t.contiguous() if t is not None else None for t in (experts, counts, valid))
    desc = _lib._balance_desc(logits, experts, valid, z_weight, reduction)
    _lib._balance_counts(logits, experts, counts)
    loss, got = BalanceFunction.apply(logits, experts, counts, valid, desc)
    return loss, (counts if counts is not None else got)


def expert_counts(experts: torch.Tensor, num_experts: int, *, valid: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Tokens per expert, int64 (B, num_experts) or (num_experts,), of experts (B, tokens, chosen) or
    (tokens, chosen); num_experts up to 1024. Entries outside [0, num_experts) are dropped slots, tokens that
    are not valid padding."""
    return _lib.apml_expert_counts(experts.contiguous(), num_experts, valid=valid.contiguous() if valid is not None else None)
