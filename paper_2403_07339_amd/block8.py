"""Linear layers and the MLP of a Transformer block in 8-bit floating point, with nothing wider kept between the passes.

Operands are e4m3 codes with a power of two for every 128 of a row (activations, gradients: blocks along the contraction) or every 128 x 128
(weights, so that a block's power of two is the same for both products they take part in):

    y      = Q(x)  Q(w)^T
    grad_x = Q(gy) Q(w)
    grad_w = Q(gy^T) Q(Q(x)^T)        (the contraction runs over the tokens: blocks along them)

What the backward pass needs of x is the operand itself, one byte an element; a power of two for a scale is why it can be turned without another
rounding (but below the smallest codes).  The MLP keeps the activation function's input in 8 bits as well and takes the slope there.
Beside ``linear.IMUnpackLinear``, whose integer products are exact: here a product takes a fraction of the time and its operands keep four significant bits.
fp32 or bfloat16, parameters alike or not; results are in x's type, gradients of parameters in theirs.
Both passes may be captured in a graph; as with every function of torch, no eager autograd graph of the same leaves may live meanwhile, or autograd would add their
gradients up on the stream where that one was made.
"""
from __future__ import annotations

import torch

from . import binding as imu


def _rows(x: torch.Tensor) -> torch.Tensor:
    return x.reshape(-1, x.shape[-1])


def _bias(b: torch.Tensor | None) -> torch.Tensor | None:
    return None if b is None else b.detach().float().contiguous()


def _pack(*blocks) -> list:
    """The tensors of some Blocks8 (or None), for save_for_backward."""
    return [t for b in blocks for t in ((b.codes, b.scales) if b is not None else (None, None))]


def _unpack(tensors, cols) -> list:
    return [imu.Blocks8(c, s, n) if c is not None else None for c, s, n in zip(tensors[::2], tensors[1::2], cols)]


def _both_ways(g: torch.Tensor, lying: bool, x) -> tuple:
    """A gradient for the products that take it: as it lies, and turned with x (None: not)."""
    if x is not None:
        (gq, gt), (_, xt) = imu.imunpack_block8_many((g, False, lying, True), x)
        return gq, gt, xt
    return imu.imunpack_block8_quantize(g)[0] if lying else None, None, None


def _empty_backward(ctx, gy, shapes):
    """Gradients of a call without rows."""
    return [torch.zeros(shape, dtype=dtype, device=gy.device) if needed else None for (shape, dtype), needed in zip(shapes, ctx.needs_input_grad)]


# (What an autograd function is told of its inputs does not know no_grad: `train` says whether anything is kept.)
class _LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, train):
        ctx.like = [(t.shape, t.dtype) if t is not None else (None, None) for t in (x, weight, bias)]
        if x.numel() == 0:
            return x.new_empty(*x.shape[:-1], weight.shape[0])
        need_x, need_w = (train and n for n in ctx.needs_input_grad[:2])
        (xq, _), (wq, turned) = imu.imunpack_block8_many((_rows(x), False, True, False), (weight, True, True, need_x))
        y = imu.imunpack_block8_gemm(xq, wq, x.dtype, _bias(bias))
        ctx.save_for_backward(*_pack(xq if need_w else None, turned))
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        (x_shape, dtype), (w_shape, w_dtype), (_, b_dtype) = ctx.like
        if gy.numel() == 0:
            return (*_empty_backward(ctx, gy, ctx.like), None)
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        xq, wt = _unpack(ctx.saved_tensors, (w_shape[1], w_shape[0]))
        g = _rows(gy)
        gx = gw = None
        gq, gt, xt = _both_ways(g, need_x, xq if need_w else None)
        if need_x:
            gx = imu.imunpack_block8_gemm(gq, wt, dtype).view(x_shape)
        if need_w:
            gw = imu.imunpack_block8_gemm(gt, xt, w_dtype)
        return gx, gw, imu.imunpack_column_sums(g).to(b_dtype) if need_b else None, None


class _MLPFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, act, gated, train):
        ctx.like = [(t.shape, t.dtype) if t is not None else (None, None) for t in (x, w1, b1, w2, b2)]
        ctx.how = act, gated
        if x.numel() == 0:
            return x.new_empty(*x.shape[:-1], w2.shape[0])
        need_x, need_w1, need_b1, need_w2 = (train and n for n in ctx.needs_input_grad[:4])
        first = need_x or need_w1 or need_b1
        (xq, _), (wq, t1), (wq2, t2) = imu.imunpack_block8_many((_rows(x), False, True, False), (w1, True, True, need_x), (w2, True, True, first))
        u = imu.imunpack_block8_gemm(xq, wq, x.dtype, _bias(b1))
        _, aq, kept = imu.imunpack_act8(u, act, gated, quantize=True, keep=first, want_y=False)
        y = imu.imunpack_block8_gemm(aq, wq2, x.dtype, _bias(b2))
        ctx.save_for_backward(*_pack(xq if need_w1 else None, t1, aq if need_w2 else None, t2, *(kept or ())))
        return y.view(*x.shape[:-1], w2.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        (x_shape, dtype), (w1_shape, w1_dtype), (_, b1_dtype), (w2_shape, w2_dtype), (_, b2_dtype) = ctx.like
        act, gated = ctx.how
        if gy.numel() == 0:
            return (*_empty_backward(ctx, gy, ctx.like), None, None, None)
        need_x, need_w1, need_b1, need_w2, need_b2 = ctx.needs_input_grad[:5]
        hidden = w2_shape[1]
        xq, t1, aq, t2, *kept = _unpack(ctx.saved_tensors, (w1_shape[1], w1_shape[0], hidden, w2_shape[0], hidden, hidden))
        g = _rows(gy)
        first = need_x or need_w1 or need_b1
        gx = gw1 = gb1 = gw2 = None
        gq, gt, at = _both_ways(g, first, aq if need_w2 else None)
        if need_w2:
            gw2 = imu.imunpack_block8_gemm(gt, at, w2_dtype)
        if first:
            gu = imu.imunpack_act8_backward(imu.imunpack_block8_gemm(gq, t2, dtype), tuple(kept), act, gated)
            gq, gt, xt = _both_ways(gu, need_x, xq if need_w1 else None)
            if need_x:
                gx = imu.imunpack_block8_gemm(gq, t1, dtype).view(x_shape)
            if need_w1:
                gw1 = imu.imunpack_block8_gemm(gt, xt, w1_dtype)
            if need_b1:
                gb1 = imu.imunpack_column_sums(gu).to(b1_dtype)
        return gx, gw1, gb1, gw2, imu.imunpack_column_sums(g).to(b2_dtype) if need_b2 else None, None, None, None


def block8_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None) -> torch.Tensor:
    """x [..., in], weight [out, in], bias [out] -> [..., out]."""
    if x.shape[-1] != weight.shape[1] or weight.numel() == 0:
        raise ValueError(f"shapes {tuple(x.shape)} and {tuple(weight.shape)} do not form x W^T")
    return _LinearFunction.apply(x, weight, bias, torch.is_grad_enabled())


def block8_mlp(x: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor, b1: torch.Tensor | None = None, b2: torch.Tensor | None = None, act: str = "gelu",
               gated: bool = False) -> torch.Tensor:
    """f(x W1^T + b1) W2^T + b2 with f GELU or SiLU; gated: f of the first half of W1's rows times the second half's product."""
    if act not in imu.ACTIVATIONS:
        raise ValueError("act is gelu or silu")
    if x.shape[-1] != w1.shape[1] or w1.numel() == 0 or w2.numel() == 0 or w1.shape[0] != w2.shape[1] * (2 if gated else 1):
        raise ValueError(f"shapes {tuple(x.shape)}, {tuple(w1.shape)} and {tuple(w2.shape)} do not form an MLP")
    return _MLPFunction.apply(x, w1, b1, w2, b2, act, gated, torch.is_grad_enabled())


class Block8Linear(torch.nn.Module):
    """``torch.nn.Linear`` with its three products in 8-bit floating point."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, device=None, dtype=torch.float32):
        super().__init__()
        ref = torch.nn.Linear(in_features, out_features, bias=bias, device=device, dtype=dtype)
        self.weight, self.bias = ref.weight, ref.bias

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return block8_linear(x, self.weight, self.bias)

    def frozen(self) -> "FrozenLinear":
        return FrozenLinear(self.weight, self.bias)


class _FrozenFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, layer):
        w = layer.weight
        ctx.like = [(x.shape, x.dtype), (None, None)]
        ctx.cols = w.cols
        ctx.save_for_backward(w.codes, w.scales)
        return layer._product(x)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        if gy.numel() == 0:
            return tuple(_empty_backward(ctx, gy, ctx.like))
        shape, dtype = ctx.like[0]
        turned = imu.imunpack_block8_turn(imu.Blocks8(*ctx.saved_tensors, ctx.cols))
        return imu.imunpack_block8_gemm(imu.imunpack_block8_quantize(_rows(gy))[0], turned, dtype).view(shape), None


class FrozenLinear:
    """A linear layer for serving: its weights are brought to 8 bits once, by this constructor, and are no parameters.  An input that requires a gradient gets it,
    Q(gy) Q(w), for which a backward pass turns the weights' codes (they are not kept both ways)."""

    @torch.no_grad()
    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None):
        self.weight, _ = imu.imunpack_block8_quantize(weight.detach(), square=True)
        self.bias = _bias(bias)

    def _product(self, x: torch.Tensor) -> torch.Tensor:
        y = imu.imunpack_block8_gemm(imu.imunpack_block8_quantize(x)[0], self.weight, x.dtype, self.bias)
        return y.view(*x.shape[:-1], self.weight.rows)

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        if x.requires_grad and torch.is_grad_enabled():
            return _FrozenFunction.apply(x, self)
        return self._product(x)


class Block8MLP(torch.nn.Module):
    """Up-projection, activation, down-projection; x, the activation function's input and its result are kept in 8 bits."""

    def __init__(self, features: int, hidden: int, act: str = "gelu", gated: bool = False, bias: bool = True, device=None, dtype=torch.float32):
        super().__init__()
        self.up = Block8Linear(features, hidden * (2 if gated else 1), bias, device, dtype)
        self.down = Block8Linear(hidden, features, bias, device, dtype)
        self.act, self.gated = act, gated

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return block8_mlp(x, self.up.weight, self.down.weight, self.up.bias, self.down.bias, self.act, self.gated)
