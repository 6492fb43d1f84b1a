"""Log probabilities of given tokens with the entropy and the largest alternatives of rows of logits, and their gradient.

    logp_t = l_t - log sum_v exp l_v,    entropy = -sum_v p_v log p_v

For scoring a text, for sampling (what was chosen and what else was likely), and as the objective of training on chosen tokens: gradients of
logp, of the entropy and of the alternatives' log probabilities go back to the logits in one pass.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as imu


class Scores(NamedTuple):
    logp: torch.Tensor | None
    entropy: torch.Tensor
    top_logp: torch.Tensor | None
    top_index: torch.Tensor | None


class _ScoresFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, top, ignore_index):
        got = imu.imunpack_logprobs(logits, tokens, top, True, ignore_index)
        ctx.save_for_backward(logits, tokens, got.stats, got.entropy, got.top_index)
        ctx.ignore_index = ignore_index
        ctx.set_materialize_grads(False)
        if got.top_index is not None:
            ctx.mark_non_differentiable(got.top_index)
        return got.logp, got.entropy, got.top_logp, got.top_index

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logp, g_entropy, g_top, _):
        logits, tokens, stats, entropy, top_index = ctx.saved_tensors
        if g_logp is None and g_entropy is None and g_top is None:
            return None, None, None, None
        saved = imu.Logprobs(None, None, stats, entropy, None, top_index)
        return imu.imunpack_logprobs_backward(logits, tokens, saved, g_logp, g_entropy, g_top, ctx.ignore_index), None, None, None


def log_probs(logits: torch.Tensor, tokens: torch.Tensor | None = None, top: int = 0, ignore_index: int = -100) -> Scores:
    """logits [..., vocab] (fp32 or bfloat16); tokens int64 [...] or [..., some to a row].  Scores of fp32: logp like tokens (0 where a token is
    ignore_index), entropy [...], top_logp and top_index (int64) [..., top], largest first, of equals the lowest place first; None where not asked for."""
    return Scores(*_ScoresFunction.apply(logits, tokens, top, ignore_index))
