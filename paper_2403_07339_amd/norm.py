"""Root-mean-square norm with the addition of the residual stream in front of it.

    h = x + residual,   y = h / sqrt(mean(h^2) + eps) * weight

What stands between the products of a Transformer block.  For training an autograd function over the library's forward and
backward kernels; for serving the output as In-Bound integers of b bits with a step per row (Sec. 4 of arXiv 2403.07339: such an
operand of the exact integer GEMM is never split).
"""
from __future__ import annotations

import torch

from . import binding as imu


class _NormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        y, h, saved = imu.imunpack_rmsnorm(x, weight, eps, residual)
        ctx.save_for_backward(*((weight, saved.rstd, h) if saved.x is None else (weight, saved.rstd, x, residual)))
        ctx.has_residual = residual is not None
        ctx.set_materialize_grads(False)
        return y, h if ctx.has_residual else None

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy, gh):
        if gy is None:
            return gh, gh, None, None
        weight, rstd, x, *residual = ctx.saved_tensors
        saved = imu.NormSaved(rstd, x, *residual) if residual else imu.NormSaved(rstd)
        gx, gw = imu.imunpack_rmsnorm_backward(gy, x, weight, saved, gh, want_weight=ctx.needs_input_grad[2])
        return gx, gx if ctx.has_residual else None, gw, None


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: torch.Tensor | None = None, eps: float = 1e-6):
    """y, or (y, h) with a residual: h = x + residual is the residual stream that goes on."""
    y, h = _NormFunction.apply(x, residual, weight, eps)
    return y if residual is None else (y, h)


class RMSNorm(torch.nn.Module):
    """``forward(x, residual=None)`` as ``rms_norm``; ``quantize(x, b, residual=None)`` the norm for serving: (q int8, scale fp32 per
    row) and, with a residual, h behind them."""

    def __init__(self, features: int, eps: float = 1e-6, device=None, dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype))
        self.eps = eps

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        return rms_norm(x, self.weight, residual, self.eps)

    @torch.no_grad()
    def quantize(self, x: torch.Tensor, b: int = 8, residual: torch.Tensor | None = None):
        q, scale, h, _ = imu.imunpack_rmsnorm_quantize(x, self.weight, self.eps, b, residual)
        return (q, scale) if residual is None else (q, scale, h)
