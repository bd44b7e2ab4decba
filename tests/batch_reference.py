"""Plain fp64 counterparts of the batch operators (pages, the 8-bit cache, attention over it, scores of tokens), with
the tolerances that their arithmetic allows."""
import math

import numpy as np

PAGE, E_MIN = 64, -100
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # of a rounding, relative to the value
OK, E_ARG, E_KV_FULL, E_CTX_OVERFLOW = 0, -1, -3, -4


def plan(seq, new, held, n_free, head, width, max_rows, free, tables):
    """One sequence after the other; all or nothing."""
    seq, new, held = (np.asarray(a, np.int64) for a in (seq, new, held))
    kv, got, tab, at, rows = seq.copy(), held.copy(), tables.copy(), head, 0
    slots, start = np.full(max_rows, -1, np.int64), np.zeros(len(seq) + 1, np.int64)
    for s in range(len(seq)):
        end = int(seq[s] + new[s])
        code = OK
        if seq[s] < 0 or new[s] < 0 or not 0 <= held[s] <= width or -(-int(seq[s]) // PAGE) > held[s]:
            code = E_ARG
        elif -(-end // PAGE) > width:
            code = E_CTX_OVERFLOW
        elif not 0 <= head <= n_free:
            code = E_ARG
        else:
            need = max(0, -(-end // PAGE) - int(held[s]))
            if at + need > n_free:
                code = E_KV_FULL
            elif rows + new[s] > max_rows:
                code = E_ARG
        if code:
            return seq, held, np.zeros(len(seq) + 1, np.int64), np.full(max_rows, -1, np.int64), tables, [code, 0, head, s]
        for _ in range(need):
            tab[s, got[s]] = free[at]
            got[s], at = got[s] + 1, at + 1
        for p in range(int(seq[s]), end):
            slots[rows] = int(tab[s, p // PAGE]) * PAGE + p % PAGE
            rows += 1
        kv[s], start[s + 1] = end, rows
    return kv, got, start, slots, tab, [OK, rows, at, -1]


def nearest_code(x):
    """The e4m3 value nearest to x, |x| <= 448: ties to even; NaN stays."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 1.0)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -6.0) - 3)
    return np.where(np.isfinite(x), np.copysign(np.rint(a / step) * step, x), np.nan)


def exponent(amax):
    """The smallest e >= E_MIN with amax <= 448 * 2**e."""
    e = E_MIN
    if amax > 0:
        e = math.frexp(amax)[1] - 10
        while amax > math.ldexp(448.0, e):
            e += 1
    return max(e, E_MIN)


class CacheModel:
    """What a cache holds, block by block: code values and exponents."""

    def __init__(self, n_pages, kv, hd):
        self.n_pages, self.kv, self.hd = n_pages, kv, hd
        self.codes = np.zeros((2, n_pages, kv, PAGE, hd))
        self.e = np.full((2, n_pages, kv), E_MIN)

    def append(self, k, v, slots):
        slots = np.asarray(slots)
        live = (slots >= 0) & (slots < self.n_pages * PAGE)
        for page in np.unique(slots[live] // PAGE):
            at = np.nonzero(live & (slots // PAGE == page))[0]
            off = slots[at] % PAGE
            fresh = bool((off == 0).any())
            for which, rows in ((0, k), (1, v)):
                for h in range(self.kv):
                    x = np.asarray(rows[at, h], np.float64)
                    fin = np.abs(x[np.isfinite(x)])
                    e = exponent(float(fin.max()) if fin.size else 0.0)
                    old = int(self.e[which, page, h])
                    if not fresh:
                        e = max(e, old)
                        if e > old:
                            self.codes[which, page, h] = nearest_code(self.codes[which, page, h] * 2.0 ** (old - e))
                    self.codes[which, page, h, off] = nearest_code(np.where(np.isfinite(x), x, np.nan) * 2.0 ** -e)
                    self.e[which, page, h] = e

    def read(self, slots):
        page, off = np.asarray(slots) // PAGE, np.asarray(slots) % PAGE
        return tuple(self.codes[w, page, :, off] * np.exp2(self.e[w, page])[..., None].astype(np.float64) for w in (0, 1))

    def sequence(self, table, length):
        p = np.arange(length)
        return self.read(np.asarray(table)[p // PAGE].astype(np.int64) * PAGE + p % PAGE)


def attention(model, q, tables, kv_lens, row_start, scale, dtype):
    """(outputs, tolerances) of the rows of every sequence; NaN tolerances mark rows of no sequence."""
    q = np.asarray(q, np.float64)
    out, tol = np.zeros(q.shape), np.full(q.shape, np.nan)
    group = q.shape[1] // model.kv
    for s in range(len(kv_lens)):
        r0, r1, length = int(row_start[s]), int(row_start[s + 1]), int(kv_lens[s])
        if r1 == r0:
            continue
        k, v = model.sequence(tables[s], length)
        for i in range(r1 - r0):
            seen = length - (r1 - r0) + i + 1
            if seen <= 0:
                tol[r0 + i] = 0.0
                continue
            for h in range(q.shape[1]):
                x, kk, vv = q[r0 + i, h], k[:seen, h // group], v[:seen, h // group]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = scale * (kk @ x)
                    size = abs(scale) * (np.abs(kk) @ np.abs(x))
                    p = np.exp(z - z.max())
                    w = p / p.sum()
                    out[r0 + i, h] = w @ vv
                    # a weight's relative error: the score's (products of up to three parts of q, summed in fp32,
                    # scaled and shifted), the exponential's, the sums' over a page and over pages, and its own
                    # rounding to 11 bits (bf16) or 22 (fp32); each enters the quotient's two sums once
                    terms = (3 * model.hd + 4) * size.max() + 4 + 2 * (80 + seen / PAGE)
                    eps = 2.0 ** -23 * terms + (2.0 ** -12 if dtype == "bf16" else 2.0 ** -22)
                    tol[r0 + i, h] = 2 * eps * (w @ np.abs(vv)) + HALF_STEP[dtype] * np.abs(out[r0 + i, h]) * (1 + 2 ** -6)
    return out, tol


def scores(z, temperature, token, n_top):
    """Of one row: (log p of the token, rank, entropy, ids, their log p)."""
    raw = np.asarray(z, np.float64) + 0.0
    order = sorted(range(len(raw)), key=lambda i: (0 if math.isnan(raw[i]) else 1, -raw[i] if not math.isnan(raw[i]) else 0, i))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        x = raw / temperature
        m = x.max()
        lp = x - m - np.log(np.exp(x - m).sum())
        p = np.exp(lp)
        h = -np.where(p > 0, p * lp, np.where(np.isnan(p), np.nan, 0.0)).sum()
    given = 0 <= token < len(raw)
    return (lp[token] if given else np.nan, order.index(token) if given else -1, h, order[:n_top], lp[order[:n_top]])


def score_tolerance(lp, V):
    """Of a log probability or an entropy: the temperature's rounding scales what is summed (|log p| and at most ln V), an
    exponential's argument has a rounding of its own, and a sum runs over 32 entries of a thread, its block and the blocks."""
    return 2.0 ** -23 * (2 * np.abs(lp) + 4 * math.log(V) + 4) + 2.0 ** -24 * (2 * 48 + V / 8192) * (1 + math.log(V))
