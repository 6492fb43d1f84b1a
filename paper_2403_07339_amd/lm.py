"""A small encoder trained on masked tokens: the layers, the norm, the loss and the optimiser of this package together.

    python -m paper_2403_07339_amd.lm [--steps N] [--state-bits 8|32] [--mlp integer|block8]

Every product of the blocks runs on the exact low-bit integer path (``linear``, ``attention``), or those of the MLP in 8-bit floating point with
activations kept that way (``block8``); between them stands ``norm.RMSNorm``,
which carries the residual stream in fp32; the head's loss over the vocabulary (``loss``) is taken where a token is masked; one call of
``optim.AdamW`` steps all parameters.  ``IntegerHead`` is the serving end: the last norm gives In-Bound integers with a step per
row, and their product with the head's weights, quantised and unpacked when they are loaded, is exact; ``score`` takes log probabilities, entropy and
alternatives from its logits (``logprobs``).
The data are synthetic: sequences that a rule continues, so that a masked token follows from its neighbours.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import binding as imu
from .attention import IMUnpackAttention
from .block8 import Block8MLP
from .linear import IMUnpackLinear, QuantConfig
from .logprobs import Scores, log_probs
from .loss import LinearCrossEntropy
from .norm import RMSNorm
from .optim import AdamW

IGNORE = -100


@dataclass
class Config:
    vocab: int = 1000
    tokens: int = 64
    width: int = 128
    hidden: int = 256
    heads: int = 4
    layers: int = 2
    mask: float = 0.15
    mlp: str = "integer"   # or "block8": 8-bit floating point


class Block(torch.nn.Module):
    """Attention and MLP, each behind a norm that also takes up what the part before added to the residual stream."""

    def __init__(self, c: Config, quant: QuantConfig, device):
        super().__init__()
        self.heads = c.heads
        self.norm1, self.norm2 = RMSNorm(c.width, device=device), RMSNorm(c.width, device=device)
        self.qkv = IMUnpackLinear(c.width, 3 * c.width, cfg=quant, device=device)
        self.out = IMUnpackLinear(c.width, c.width, cfg=quant, device=device)
        if c.mlp == "block8":
            self.mlp = Block8MLP(c.width, c.hidden, device=device)
        elif c.mlp == "integer":
            self.up = IMUnpackLinear(c.width, c.hidden, cfg=quant, device=device)
            self.down = IMUnpackLinear(c.hidden, c.width, cfg=quant, device=device)
        else:
            raise ValueError("mlp is integer or block8")
        self.eight = c.mlp == "block8"
        self.attention = IMUnpackAttention(quant)

    def forward(self, x: torch.Tensor, stream: torch.Tensor):
        y, stream = self.norm1(x, stream)
        b, t, w = y.shape
        q, k, v = self.qkv(y).view(b, t, 3, self.heads, w // self.heads).permute(2, 0, 3, 1, 4).contiguous()  # (one batch of products, not a loop of them)
        x = self.out(self.attention(q, k, v).transpose(1, 2).reshape(b, t, w))
        y, stream = self.norm2(x, stream)
        if self.eight:
            return self.mlp(y), stream
        return self.down(torch.nn.functional.gelu(self.up(y))), stream


class MaskedLM(torch.nn.Module):
    """``forward(tokens, target)``: the mean loss where target is not IGNORE.  ``encode(tokens)``: what the last block adds and the
    residual stream, which the last norm brings together."""

    def __init__(self, c: Config, quant: QuantConfig | None = None, device="cuda"):
        super().__init__()
        # (steps from the largest entry: the gradient of a matrix of attention weights is next to nothing but where a masked token looks at a few others, so
        # that any percentile below may lie further under its largest entry than 32-bit integers reach, and the product refuses it)
        quant = quant or QuantConfig(beta_x=255.0, beta_w=255.0, beta_g=1023.0, p=100.0, strategy_a=imu.ROW, strategy_b=imu.COL)
        self.embed = torch.nn.Embedding(c.vocab + 1, c.width, device=device)   # the last one stands for a masked token
        self.place = torch.nn.Parameter(0.02 * torch.randn(c.tokens, c.width, device=device))
        self.blocks = torch.nn.ModuleList(Block(c, quant, device) for _ in range(c.layers))
        self.norm = RMSNorm(c.width, device=device)
        self.head = LinearCrossEntropy(c.width, c.vocab, ignore_index=IGNORE, device=device)

    def encode(self, tokens: torch.Tensor):
        x, stream = self.embed(tokens), self.place[: tokens.shape[1]].expand(*tokens.shape, -1)
        for block in self.blocks:
            x, stream = block(x, stream)
        return x, stream

    def forward(self, tokens: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        return self.head(self.norm(*self.encode(tokens))[0], target)


class IntegerHead:
    """Logits for serving: the norm's rows as In-Bound integers of b bits, the head's weights as RTN integers whose heavy hitters are
    unpacked, their product exact (and the weights' unpacking kept from call to call)."""

    def __init__(self, model: MaskedLM, b: int = 8):
        self.norm, self.b, weight = model.norm, b, model.head.weight.detach()
        self.step = float((4.0 * weight.double().std(unbiased=False) / (2 ** b - 1)).float())
        self.Q, self.stats, _ = imu.imunpack_quantize(weight, self.step, b, want_ob_list=True)
        self.plan = imu.Plan()
        self.stored = None

    def __call__(self, x: torch.Tensor, stream: torch.Tensor) -> torch.Tensor:
        q, scale, _ = self.norm.quantize(x, self.b, stream)
        rows = q.view(-1, q.shape[-1]).to(torch.int32)
        imu.imunpack_plan(rows, self.Q, self.b, imu.ROW, imu.BOTH, None, self.stats, self.plan)
        need = self.plan.unpacked_bytes()[1]
        if self.stored is None or self.stored.numel() < need:
            self.stored = torch.empty(need, dtype=torch.int8, device=rows.device)
        a, b = imu.imunpack_unpack(self.plan, rows, self.Q, None, self.stored)
        out = torch.empty(rows.shape[0], self.Q.shape[0], dtype=torch.float32, device=rows.device)
        imu.imunpack_gemm(self.plan, a, b, 1.0, self.step, None, out)
        self.plan.keep_weights()   # from here on the plan has an unpacking to keep
        return (out * scale.view(-1, 1)).view(*x.shape[:-1], -1)


@torch.no_grad()
def score(model: MaskedLM, head: IntegerHead, tokens: torch.Tensor, target: torch.Tensor, top: int = 5) -> Scores:
    """Log probabilities of target under the integer head (0 where it is IGNORE), the entropy of every position and its `top` likeliest tokens."""
    return log_probs(head(*model.encode(tokens)), target, top, IGNORE)


def batch(c: Config, sequences: int, generator: torch.Generator, device="cuda"):
    """(tokens, target): sequences a, a + s, a + 2 s, ... modulo the vocabulary with s of a few steps; some tokens masked."""
    start = torch.randint(0, c.vocab, (sequences, 1), generator=generator)
    step = torch.randint(1, 4, (sequences, 1), generator=generator)
    tokens = (start + step * torch.arange(c.tokens)) % c.vocab
    hidden = torch.rand(tokens.shape, generator=generator) < c.mask
    target = torch.where(hidden, tokens, IGNORE)
    return torch.where(hidden, c.vocab, tokens).to(device), target.to(device)


def train(c: Config, steps: int, sequences: int = 32, lr: float = 3e-3, state_bits: int = 8, seed: int = 0, tell=None):
    """A model after so many steps, and the loss of each."""
    torch.manual_seed(seed)
    model = MaskedLM(c)
    optimizer = AdamW(model.parameters(), lr=lr, weight_decay=0.01, state_bits=state_bits, seed=seed)
    generator = torch.Generator().manual_seed(seed)
    losses = []
    for k in range(steps):
        loss = model(*batch(c, sequences, generator))
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
        if tell and (k % 10 == 0 or k + 1 == steps):
            tell(f"step {k:4d}  loss {float(losses[-1]):.4f}")
    return model, torch.stack(losses).cpu() if losses else torch.empty(0)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--sequences", type=int, default=32)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--mlp", default="integer", choices=("integer", "block8"))
    a = ap.parse_args()
    c = Config(mlp=a.mlp)
    model, _ = train(c, a.steps, a.sequences, state_bits=a.state_bits, tell=lambda s: print(s, flush=True))
    tokens, target = batch(c, 64, torch.Generator().manual_seed(1))
    got = score(model, IntegerHead(model), tokens, target)
    at = target != IGNORE
    print(f"masked tokens guessed from the integer head's logits: {float((got.top_index[..., 0][at] == target[at]).float().mean()):.3f}, "
          f"among the first five {float((got.top_index[at] == target[at][:, None]).any(-1).float().mean()):.3f}; "
          f"log probability {float(got.logp[at].mean()):.3f}, entropy {float(got.entropy[at].mean()):.3f}")


if __name__ == "__main__":
    main()
