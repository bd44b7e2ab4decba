"""The vocabulary head's loss and its gradient in 64 bits, with the tolerances that the kernels' arithmetic allows."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def chain(n, dtype):
    """Of a product's sum over n terms, relative to the sum of magnitudes: 32 terms meet in a matrix instruction and are
    added to what is there; fp32 operands enter as six such products of parts, and what the other three would add (a number cut off at
    8 bits leaves less than 2^-7 of it: the parts are below 1, 2^-7 and 2^-14 of it)."""
    return 2.0 ** -23 * (n / 32 + 33) * (1 if dtype == torch.bfloat16 else 6) + (2 * 2.0 ** -21 + 2.0 ** -28 if dtype == torch.float32 else 0.0)


class Reference:
    def __init__(self, hidden, head, targets, weights=None):
        self.dtype, self.V = hidden.dtype, head.shape[0]
        self.h, self.w, self.t = hidden.double(), head.double(), targets.long()
        self.trained = (self.t >= 0) & (self.t < self.V)
        self.g = torch.ones(len(self.t), dtype=torch.float64, device=hidden.device) if weights is None else weights.double()
        self.kept = self.trained & (self.g != 0)
        at = torch.where(self.trained, self.t, 0)[:, None]
        z = self.h @ self.w.t()
        size = self.h.abs() @ self.w.abs().t()
        self.z_tol = chain(hidden.shape[1], self.dtype) * size
        m = z.amax(1, keepdim=True)
        self.lse = (m + (z - m).exp().sum(1, keepdim=True).log())[:, 0]
        worst = self.z_tol.amax(1)
        # an exponential's argument is off by its own rounding (its mean under softmax is at most ln V), the sum has the
        # tile's, the block's and the tiles' terms, then the result's rounding
        self.lse_tol = worst + 2.0 ** -23 * (2 * math.log(self.V) + 60 + self.V / 256 / 64) + 2.0 ** -23 * (self.lse.abs() + worst)
        self.loss = torch.where(self.trained, self.lse - z.gather(1, at)[:, 0], 0.0)
        self.loss_tol = torch.where(self.trained, self.lse_tol + worst + 2.0 ** -23 * self.loss.abs(), 0.0)
        q = z - self.lse[:, None]
        p = q.exp()
        one = torch.zeros_like(p).scatter_(1, at, 1.0) * self.trained[:, None]
        g = torch.where(self.kept, self.g, 0.0)[:, None]
        keep = self.kept[:, None]
        self.dz = torch.where(keep, g * (p - one), 0.0)
        # p's relative error is that of its argument; then dz's rounding
        arg = self.z_tol + self.lse_tol[:, None] + 2.0 ** -23 * (q.abs() + 8)
        tol = torch.where(keep, g.abs() * p * arg * (1 + arg), 0.0)
        self.dz_tol = tol + (HALF_STEP[self.dtype] + 2.0 ** -23) * (self.dz.abs() + tol)

    def _product(self, dz, tol, x, n):
        want = dz @ x
        bound = tol @ x.abs() + chain(n, self.dtype) * ((dz.abs() + tol) @ x.abs())
        return want, bound + HALF_STEP[self.dtype] * (want.abs() + bound) + 1e-37

    def d_hidden(self):
        w = self.w
        return self._product(self.dz, self.dz_tol, w, self.V + 32 * 256)     # (up to 256 parts are added up)

    def d_head(self):
        h = torch.where(self.kept[:, None], self.h, 0.0)
        return self._product(self.dz.t().contiguous(), self.dz_tol.t().contiguous(), h, h.shape[0])


def inputs(M, V, K, dtype, seed, device="cuda", scale=1.0):
    """Rows and a head with logits of a few units, targets some of which are left out, weights some of which are 0."""
    g = torch.Generator(device=device).manual_seed(seed)
    hidden = torch.randn(M, K, device=device, generator=g)
    head = torch.randn(V, K, device=device, generator=g) * (2.0 * scale / math.sqrt(K))
    targets = torch.randint(0, V, (M,), device=device, generator=g)
    hidden[::3] += head[targets[::3]] * (math.sqrt(K) / 2)
    out = torch.rand(M, device=device, generator=g)
    targets = torch.where(out < 0.1, -1, torch.where(out < 0.15, V, targets))
    weights = torch.rand(M, device=device, generator=g) + 0.5
    weights[out > 0.93] = 0.0
    return hidden.to(dtype), head.to(dtype), targets.int(), weights
