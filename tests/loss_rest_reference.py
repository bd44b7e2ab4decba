"""Inputs whose targets' dz bf16 rounds by nearly half a step, all to the same side, and the tolerance of a dW that has
back what that rounding took."""
import math

import torch

from tests.loss_reference import HALF_STEP, Reference

STEP = 2.0 ** -8      # half of bf16's step between 1 and 2


class RestReference(Reference):
    """dz of a row's target reaches dW in two bf16 numbers: what the second leaves is half a step of half a step.  All else
    as in Reference."""

    def d_head_tol(self):
        half = HALF_STEP[self.dtype]
        tol = (self.dz_tol - (half + 2.0 ** -23) * self.dz.abs()) / (1 + half + 2.0 ** -23)      # (before dz is rounded)
        at = torch.where(self.trained, self.t, 0)[:, None]
        target = torch.zeros_like(self.dz).scatter_(1, at, 1.0) * self.kept[:, None]
        lost = torch.where(target > 0, half * half, half)
        tol = tol + (lost + 2.0 ** -23) * (self.dz.abs() + tol)
        h = torch.where(self.kept[:, None], self.h, 0.0)
        return self._product(self.dz.t().contiguous(), tol.t().contiguous(), h, 2 * h.shape[0])    # (the remainders are as many terms more)


def half_step_inputs(M, V, K, seed, same=0, device="cuda"):
    """bf16 rows of nearly equal logits, so that p is about 1 / V, and weights that make dz of a target -1.25 - 2^-8 c, c in
    (0.8, 0.97) (not -1, whose products with hidden are bf16 numbers).  same: targets are of that many entries only."""
    g = torch.Generator(device=device).manual_seed(seed)
    hidden = torch.randn(M, K, device=device, generator=g).to(torch.bfloat16)
    head = (torch.randn(V, K, device=device, generator=g) * (0.01 / math.sqrt(K))).to(torch.bfloat16)
    targets = torch.randint(0, V, (M,), device=device, generator=g)
    if same:
        targets = torch.randint(0, V, (same,), device=device, generator=g)[torch.randint(0, same, (M,), device=device, generator=g)]
    weights = (1.25 + STEP * (0.8 + 0.17 * torch.rand(M, device=device, generator=g))) / (1 - 1.0 / V)
    out = torch.rand(M, device=device, generator=g)
    targets = torch.where(out < 0.06, -1, torch.where(out < 0.1, V, targets))
    weights[out > 0.95] = 0.0
    return hidden, head, targets.int(), weights
