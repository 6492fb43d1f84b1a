"""Softmax cross entropy of a linear head over a vocabulary, without keeping the logits.

    loss_t = log sum_v exp(x_t . W_v) - x_t . W_target(t)

The head's product and its two gradients run inside the library, a piece of the rows at a time; the gradients of a mean or a sum are made
by the forward pass, while the product is there, and multiplied with what arrives from above by the backward pass.  Where none will be
asked for (``torch.no_grad``, operands without ``requires_grad``) the loss alone is taken.  Rows whose target is
``ignore_index`` take no part.  fp32 or bfloat16 (both operands alike).
"""
from __future__ import annotations

import math

import torch

from . import binding as imu


class _LossFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target, ignore_index, reduction):
        want = ctx.needs_input_grad[:2]
        loss, ctx.saved = imu.imunpack_xent(x, weight, target, ignore_index, reduction, any(want), *want)
        if any(want):
            ctx.save_for_backward(x, weight, target)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        gx, gw = imu.imunpack_xent_backward(*ctx.saved_tensors, ctx.saved, grad, *ctx.needs_input_grad[:2])
        return gx, gw, None, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """x [..., d], weight [vocab, d], target int64 [...]: the mean (over rows with a target; 0 if there are none), the sum, or with
    "none" the loss of every row, in fp32."""
    if not (torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad)):  # (what an autograd function is told of its inputs does not know no_grad)
        return imu.imunpack_xent(x, weight, target, ignore_index, reduction)[0]
    return _LossFunction.apply(x, weight, target, ignore_index, reduction)


class LinearCrossEntropy(torch.nn.Module):
    """A head of ``vocab`` rows of ``features`` with its loss: ``forward(x, target)``."""

    def __init__(self, features: int, vocab: int, ignore_index: int = -100, reduction: str = "mean", device=None, dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(vocab, features, device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, std=1.0 / math.sqrt(features))
        self.ignore_index, self.reduction = ignore_index, reduction

    def forward(self, x: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        return linear_cross_entropy(x, self.weight, target, self.ignore_index, self.reduction)
