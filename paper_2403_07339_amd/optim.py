"""AdamW whose step over all parameters of a group is one call of the library, with states in 32 or in 8 bits."""
from __future__ import annotations

import torch

from . import binding as imu


def _capturing() -> bool:
    return torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing()


class AdamW(torch.optim.Optimizer):
    """Decoupled weight decay, bias-corrected averages, fp32 parameters (``state_bits``: 32, or 8 for e4m3 codes of the first
    average and of the root of the second with a scale per 256 elements; ``seed``: of the rounding of 8-bit states).
    Parameters whose ``grad`` is None are left out of a step.  ``copies``: a dict from parameters to bfloat16 tensors that
    every step refreshes (working copies for a product in bfloat16; a gradient of theirs is not read).
    A step is not for capture in a graph, which would repeat its number and its random bits."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, state_bits: int = 32,
                 seed: int = 0, copies: dict | None = None):
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        if not lr >= 0.0 or not eps >= 0.0 or not weight_decay >= 0.0 or not all(0.0 <= b < 1.0 for b in betas):
            raise ValueError("lr, eps, weight_decay not negative, betas in [0, 1)")
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))
        self.state_bits, self.seed, self.copies = state_bits, seed, copies or {}

    def _state(self, p):
        st = self.state[p]
        if not st:
            st["step"] = 0
            if self.state_bits == 32:
                st["exp_avg"], st["exp_avg_sq"] = (torch.zeros_like(p, memory_format=torch.contiguous_format) for _ in range(2))
            else:
                blocks = -(-p.numel() // imu.ADAMW_BLOCK)
                for name in ("exp_avg", "exp_avg_sq"):
                    st[name] = torch.zeros(blocks * imu.ADAMW_BLOCK, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                    st[name + "_scale"] = torch.zeros(blocks, dtype=torch.float32, device=p.device)
        return st

    def load_state_dict(self, state_dict):
        """As torch.optim.Optimizer, which turns states into the parameters' type; codes become codes again (exactly).  States of the other
        width are refused: their numbers mean something else."""
        for st in state_dict["state"].values():
            if ("exp_avg_scale" in st) != (self.state_bits == 8):
                raise ValueError(f"the states to load have {8 if 'exp_avg_scale' in st else 32} bits, this optimiser's {self.state_bits}")
        super().load_state_dict(state_dict)
        if self.state_bits == 8:
            for st in self.state.values():
                for name in ("exp_avg", "exp_avg_sq"):
                    st[name] = st[name].to(torch.float8_e4m3fn)

    @torch.no_grad()
    def step(self, closure=None):
        if _capturing():
            raise RuntimeError("a step of AdamW cannot be captured: a graph would repeat its number and its random bits")
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for index, group in enumerate(self.param_groups):
            calls: dict = {}   # parameters that have taken as many steps, with gradients of one type and a copy or none, go together
            for p in group["params"]:
                if p.grad is None:
                    continue
                st = self._state(p)
                calls.setdefault((st["step"] + 1, p.grad.dtype, p in self.copies), []).append((p, st))
            for number, ((step, _, copied), some) in enumerate(calls.items()):
                ps, sts = [p for p, _ in some], [s for _, s in some]
                eight = self.state_bits == 8
                dense = [p.data if p.is_contiguous() else p.data.contiguous() for p in ps]
                imu.imunpack_adamw(dense, [p.grad.contiguous() for p in ps], [s["exp_avg"] for s in sts], [s["exp_avg_sq"] for s in sts], step,
                                   lr=group["lr"], beta1=group["betas"][0], beta2=group["betas"][1], eps=group["eps"], weight_decay=group["weight_decay"],
                                   m_scales=[s["exp_avg_scale"] for s in sts] if eight else None, v_scales=[s["exp_avg_sq_scale"] for s in sts] if eight else None,
                                   copies=[self.copies[p] for p in ps] if copied else None, seed=self.seed + 0x10001 * index + 0x3C6EF35F * number)
                for p, q, st in zip(ps, dense, sts):
                    st["step"] = step
                    if not p.is_contiguous():
                        p.data.copy_(q)
                torch.autograd.graph.increment_version(ps + [self.copies[p] for p in ps] if copied else ps)  # (the library writes past autograd)
        return loss
