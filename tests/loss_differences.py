"""The head loss along lines on which its slope is large, in 64 bits: what its differences and its gradient may be apart by.

Between two points x+ and x- about x the loss changes by the gradient at x times (x+ - x-) and a rest that 64 bits give
exactly; what a kernel's losses and gradient leave beside that is their own rounding."""
import torch

from tests.loss_reference import Reference, inputs


class Line:
    """which: 0 hidden, 1 head.  The line runs along the gradient's entries in a random half of the places."""

    def __init__(self, which, dtype, seed, M=60, V=400, K=128, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        hidden, head, targets, self.weights = inputs(M, V, K, dtype, seed, device=device)
        self.targets = targets.clamp(0, V - 1)
        self.middle, self.which = (hidden, head), which
        ref = Reference(hidden, head, self.targets, self.weights)
        gradient, gradient_tol = (ref.d_hidden, ref.d_head)[which]()
        d = gradient * (torch.rand(gradient.shape, device=device, generator=g) < 0.5)
        d = 0.25 * d / d.norm()
        x = self.middle[which]
        self.ends = [(x.double() + sign * d).to(dtype) for sign in (1, -1)]
        self.step = self.ends[0].double() - self.ends[1].double()      # (what the type makes of it)
        refs = [Reference(*self.at(e), self.targets, self.weights) for e in self.ends]
        true = [float((r.loss * self.weights.double()).sum()) for r in refs]
        self.rise = float((gradient * self.step).sum())
        self.rest = true[0] - true[1] - self.rise
        self.allowed = sum(float((r.loss_tol * self.weights.double()).sum()) for r in refs) + float((gradient_tol * self.step.abs()).sum())
        self.gradient = gradient

    def at(self, x):
        return (x, self.middle[1]) if self.which == 0 else (self.middle[0], x)

    def off(self, losses, gradient):
        """How far the losses at the two ends are from what the gradient says."""
        total = [float((x.double() * self.weights.double()).sum()) for x in losses]
        return abs(total[0] - total[1] - float((gradient.double() * self.step).sum()) - self.rest)
