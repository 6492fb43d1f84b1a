"""Softmax cross entropy of a linear head over a vocabulary, without keeping the logits.

    loss_t = log sum_v exp(x_t . W_v) - x_t . W_target(t)

The head's product and its two gradients run inside the library, a piece of the vocabulary at a time; rows whose target is
``ignore_index`` take no part.  fp32 or bfloat16 (both operands alike).
"""
from __future__ import annotations

import math

import torch

from . import binding as imu


class _LossFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target, ignore_index, reduction):
        wanted = ctx.needs_input_grad[0] or ctx.needs_input_grad[1]
        loss, saved = imu.imunpack_xent(x, weight, target, ignore_index, reduction, want_grad=wanted)
        if wanted:
            ctx.save_for_backward(x, weight, target, saved.buffer)
            ctx.saved = (saved.backward_bytes, reduction)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, target, buffer = ctx.saved_tensors
        gx, gw = imu.imunpack_xent_backward(x, weight, target, imu.XentSaved(buffer, *ctx.saved), grad, ctx.needs_input_grad[0], ctx.needs_input_grad[1])
        return gx, gw, None, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """x [..., d], weight [vocab, d], target int64 [...]: the mean (over rows with a target; 0 if there are none), the sum, or with
    "none" the loss of every row, in fp32."""
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
