"""Inputs of the fp32 head loss whose numbers have large second and third bf16 parts (mantissas of ones) and whose results
are single products, with tolerances near 2^-19: what the six products of parts that are made leave out, and no more.

A number cut off at 8 bits leaves less than 2^-7 of it: parts are below 1, 2^-7 and 2^-14 of it, the three products left out
below 2^-21, 2^-21 and 2^-28.  The six are added in fp32, each with an error of at most 2^-23 of the sum (zeros add none)."""
import math

import torch

REL = 2 * 2.0 ** -21 + 2.0 ** -28 + 6 * 2.0 ** -23 * (1 + 2.0 ** -6)
SIX = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]


def ones(shape, g, exponents, signs=True, device="cuda"):
    """(2 - 2^-23) 2^e, of either sign."""
    e = torch.tensor(exponents, device=device)[torch.randint(0, len(exponents), shape, device=device, generator=g)]
    x = torch.ldexp(torch.full(shape, 2 - 2.0 ** -23, device=device), e)
    return torch.where(torch.rand(shape, device=device, generator=g) < 0.5, -x, x) if signs else x


def parts(x):
    """Three bf16 numbers that sum to the fp32 x, cut off."""
    out, rest = [], x
    for _ in range(3):
        p = (rest.view(torch.int32) & -65536).view(torch.float32)
        out.append(p.double())
        rest = rest - p
    return out


def product(x, y, which=SIX):
    """x y, of the products of parts that `which` lists."""
    a, b = parts(x.contiguous()), parts(y.contiguous())
    return sum(a[i] * b[j] for i, j in which)


class Scores:
    """Rows of hidden with one number each, so that a logit is one product."""

    def __init__(self, M, V, K, seed, big, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.at = torch.randperm(K, device=device, generator=g)[:M] if M <= K else torch.randint(0, K, (M,), device=device, generator=g)
        self.x = ones((M,), g, [4 if big else 2], device=device)
        self.hidden = torch.zeros(M, K, device=device)
        self.hidden[torch.arange(M, device=device), self.at] = self.x
        self.head = ones((V, K), g, [4, 5] if big else [1, 2], device=device)
        self.targets = torch.randint(0, V, (M,), device=device, generator=g).int()
        self.weights = torch.rand(M, device=device, generator=g) + 0.5
        self.w = self.head[:, self.at].t().contiguous()      # [row][entry]: the numbers that the row's meets
        self.z = self.x.double()[:, None] * self.w.double()
        self.lse = self.z.logsumexp(1)

    def emulated(self, which=SIX):
        """(lse, loss) and the gradient of the head at the rows' columns, of logits of these products of parts."""
        z = product(self.x[:, None].expand_as(self.w), self.w, which)
        lse = z.logsumexp(1)
        one = torch.zeros_like(z).scatter_(1, self.targets.long()[:, None], 1.0)
        dz = self.weights.double()[:, None] * ((z - self.lse.float().double()[:, None]).exp() - one)
        return (lse.float(), (lse - z.gather(1, self.targets.long()[:, None])[:, 0]).float()), (dz * self.x.double()[:, None]).float()

    def scores_off(self, lse, loss):
        """The largest errors of (lse, loss), over their tolerances."""
        V, t = self.z.shape[1], self.targets.long()[:, None]
        most, zt = self.z.abs().amax(1), self.z.gather(1, t)[:, 0]
        tol = REL * most + 2.0 ** -23 * (2 * math.log(V) + 60 + V / 16384 + self.lse.abs())
        want = self.lse - zt
        tol_loss = tol + REL * zt.abs() + 2.0 ** -23 * want.abs()
        return float(((lse.double() - self.lse).abs() / tol).max()), float(((loss.double() - want).abs() / tol_loss).max())

    def head_gradient_off(self, dw):
        """The same of d_head at the rows' columns (as [row][entry]; one row each), with `lse` rounded to fp32."""
        lse = self.lse.float().double()[:, None]
        q = self.z - lse
        p, one = q.exp(), torch.zeros_like(q).scatter_(1, self.targets.long()[:, None], 1.0)
        g = self.weights.double()[:, None]
        want = g * (p - one) * self.x.double()[:, None]
        # the argument's error, the exponential's and its difference's, the weight's product; then the product with hidden
        arg = REL * self.z.abs() + 2.0 ** -23 * (q.abs() + 8)
        tol = g * p * arg * (1 + arg) * self.x.double().abs()[:, None] + want.abs() * (REL + 2.0 ** -22) + 1e-36
        return float(((dw.double() - want).abs() / tol).max())


class Gradients:
    """One entry of the vocabulary has all of the probability and every row another target: dz is -weight there, and the
    gradients at a row's target and of a row are single products."""

    def __init__(self, M, V, K, seed, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        down = max(0, math.ceil(math.log2(4 * K / 200)))      # |logits| of at most 200, for one of 512
        self.hidden, self.head = ones((M, K), g, [-1, 0], device=device), ones((V, K), g, [-down, -down - 1], device=device)
        self.free = int(torch.randint(0, K, (1,), device=device, generator=g))
        self.hidden[:, self.free], self.head[:, self.free] = 8.0, 0.0
        self.head[V - 1] = 0.0
        self.head[V - 1, self.free] = 64.0
        self.targets = torch.randperm(V - 1, device=device, generator=g)[:M].int()
        self.weights = ones((M,), g, [-3, -2, -1, 0], signs=False, device=device)
        self.lse = torch.full((M,), 512.0, device=device)
        self.columns = torch.arange(K, device=device) != self.free

    def emulated(self, which=SIX):
        """(d_hidden without the free column, d_head at the targets), of these products of parts."""
        g, w = self.weights[:, None], self.head[self.targets.long()]
        return -product(g.expand_as(w), w, which)[:, self.columns].float(), -product(g.expand_as(self.hidden), self.hidden, which).float()

    def off(self, dh, dw):
        g = self.weights.double()[:, None]
        want = (-g * self.head[self.targets.long()].double())[:, self.columns], -g * self.hidden.double()
        return tuple(float(((a.double() - b).abs() / (b.abs() * (REL + 2.0 ** -24))).max()) for a, b in zip((dh, dw), want))
