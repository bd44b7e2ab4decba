"""Operators for a batch of requests over one paged 8-bit cache, as cases that can be timed and compared.

A case is a dict of plain values.  Four kinds, each one call (an append: the call and its reading back) of
paper_2606_03113_amd.lede:

  plan     op_cache_plan: block tables and the slot map of a pass, from the requests' lengths
  append   op_cache_append of K/V rows at their slots, and op_cache_read of every page that they touched
  attend   op_cache_attention of query rows of ragged sequences
  score    op_logprobs of given tokens, with their ranks, the entropy and the top alternatives

`run` computes them in elementary torch operations, or, where `own` is true, by those calls.

The cache holds e4m3 codes with one power-of-two scale for each (page of 64 tokens, KV head), for keys and for
values: a region of key codes [page][head][64][dim], value codes [page][head][dim][64] and scale words [page][head][2]
(keys, values), a word being the exponent plus 127, and 256 more where the block holds a NaN.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
E_MIN = -100            # the smallest scale is 2**E_MIN
NAN_BIT = 256
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# (query heads, KV heads, head dim) of the repository's workloads, and a wide group
HEADS = [(4, 4, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (28, 4, 128), (16, 2, 64)]
ATTEND_FLOPS = 1.5e11   # of a drawn attention
ATTEND_BYTES = 6e8
SCORE_VALUES = 2048 * 128256


def listed():
    return [
        # one token more for each of a batch of requests: the smallest call, before every decoding step
        {"name": "plan-step", "kind": "plan", "seqs": 64, "new_lo": 1, "new_hi": 1, "cached": 4096},
        # prompts of a full server at once, some of them further turns
        {"name": "plan-prompts", "kind": "plan", "seqs": 500, "new_lo": 0, "new_hi": 511, "cached": 2000},
        # a decoding step's keys and values of a batch, grouped heads
        {"name": "append-step", "kind": "append", "dtype": "bf16", "kv": 8, "hd": 128, "seqs": 48, "new": 1, "cached": 4000},
        # a prompt's keys and values, one KV head for each query head
        {"name": "append-prompt", "kind": "append", "dtype": "bf16", "kv": 32, "hd": 128, "seqs": 3, "new": 2731, "cached": 130},
        # fp32 rows of five verify positions each, 64-wide heads
        {"name": "append-verify", "kind": "append", "dtype": "f32", "kv": 4, "hd": 64, "seqs": 17, "new": 5, "cached": 700},
        # the smallest attention: one token of the smallest model behind a short prompt, fp32
        {"name": "attend-tiny", "kind": "attend", "dtype": "f32", "q": 4, "kv": 4, "hd": 64, "seqs": 1, "new": 1, "ctx": 96},
        # the ordinary one: a decoding step of a batch with ragged contexts, grouped heads
        {"name": "attend-step", "kind": "attend", "dtype": "bf16", "q": 32, "kv": 8, "hd": 128, "seqs": 64, "new": 1, "ctx": 6000},
        # drafts verified behind very long contexts: few rows, a long axis
        {"name": "attend-long", "kind": "attend", "dtype": "bf16", "q": 64, "kv": 8, "hd": 128, "seqs": 2, "new": 5, "ctx": 131000},
        # prompts in chunks behind cached ones: many rows
        {"name": "attend-chunk", "kind": "attend", "dtype": "bf16", "q": 32, "kv": 32, "hd": 128, "seqs": 3, "new": 1000, "ctx": 4100},
        # an fp32 chunk of odd sizes
        {"name": "attend-f32", "kind": "attend", "dtype": "f32", "q": 32, "kv": 8, "hd": 128, "seqs": 5, "new": 77, "ctx": 1500},
        # the rows of one verify pass: the drafts' log probabilities and the exit policy's five alternatives
        {"name": "score-step", "kind": "score", "dtype": "f32", "rows": 5, "vocab": 32000, "top": 5, "temperature": 0.6},
        # a prompt's tokens over the largest vocabulary
        {"name": "score-prompt", "kind": "score", "dtype": "bf16", "rows": 2048, "vocab": 128256, "top": 20, "temperature": 1.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "score", "score"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "plan":
        seqs = _log_int(rng, 1, 1500)
        hi = _log_int(rng, 1, 125000 // seqs)
        return {"kind": kind, "seqs": seqs, "new_lo": rng.choice([0, 1, hi]), "new_hi": hi, "cached": _log_int(rng, 1, 8000)}
    if kind == "score":
        vocab = _log_int(rng, 100, 200000)
        return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, min(4096, SCORE_VALUES // 2 // vocab)), "vocab": vocab,
                "top": rng.choice([0, 1, rng.randint(1, 32)]), "temperature": rng.choice([1.0, 1.0, 0.6, 1.7])}
    q, kv, hd = rng.choice(HEADS)
    if kind == "append":
        seqs = _log_int(rng, 1, 256)
        return {"kind": kind, "dtype": dtype, "kv": kv, "hd": hd, "seqs": seqs, "new": _log_int(rng, 1, max(1, 4096 // seqs)),
                "cached": _log_int(rng, 1, 4000)}
    shape = rng.choice(["step", "verify", "chunk", "long"])
    seqs = 1 if shape == "long" else _log_int(rng, 1, 16 if shape == "chunk" else 128)
    new = 1 if shape == "step" else _log_int(rng, 2, 16) if shape in ("verify", "long") else _log_int(rng, 17, 2048)
    most = min(ATTEND_BYTES / (2.0 * seqs * kv * hd), ATTEND_FLOPS / (4.0 * q * hd * seqs * new)) - new
    lo, hi = (20000, 200000) if shape == "long" else (1, 16000)
    new = max(1, new if most > 1 else int(ATTEND_FLOPS / (4.0 * q * hd * seqs) / 2048))
    return {"kind": kind, "dtype": dtype, "q": q, "kv": kv, "hd": hd, "seqs": seqs, "new": new,
            "ctx": max(1, min(int(max(most, 1)), _log_int(rng, lo, hi)))}


# ---- inputs ----------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to("cuda")


def _lengths(case):
    """Cached and new tokens of every sequence, the case's own: ragged, and of eight or more one has nothing new."""
    r = np.random.default_rng(11)
    n = case["seqs"]
    if case["kind"] == "plan":
        cached = r.integers(0, case["cached"] + 1, n)
        new = r.integers(case["new_lo"], case["new_hi"] + 1, n)
        return cached, new
    ctx = case.get("ctx", case.get("cached"))
    cached = r.integers(ctx // 2, ctx + 1, n) if n > 1 else np.array([ctx])
    new = r.integers((case["new"] + 1) // 2, case["new"] + 1, n) if n > 1 else np.array([case["new"]])
    if n >= 8 and case["kind"] == "attend":
        new[n // 2] = 0
    return cached, new


def _tables(held, width, r, spare=3):
    """Tables of distinct pages in random order, the pool's size, and the pages left over."""
    total = int(held.sum())
    order = r.permutation(total + spare)
    tables = np.full((len(held), width), -1, np.int32)
    at = 0
    for s, h in enumerate(held):
        tables[s, :h] = order[at:at + h]
        at += h
    return tables, total + spare, order[at:].astype(np.int32)


def _region(n_pages, kv, hd, g):
    """A cache of random contents: normal values whose blocks differ in size, as heads and pages do."""
    size = n_pages * kv * PAGE * hd
    region = torch.empty(2 * size + n_pages * kv * 8, dtype=torch.uint8, device="cuda")
    step = 1 << 26
    for at in range(0, 2 * size, step):
        m = min(step, 2 * size - at)
        x = torch.empty(m, dtype=torch.float32, device="cuda").normal_(0.0, 90.0, generator=g).clamp_(-448.0, 448.0)
        region[at:at + m] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    words = torch.randint(127 - 8, 127 - 5, (n_pages * kv * 2,), device="cuda", generator=g, dtype=torch.int32)
    region[2 * size:] = words.view(torch.uint8)
    return region


def _parts(region, n_pages, kv, hd):
    """Key codes [page][head][64][dim], value codes [page][head][dim][64] and scale words [page][head][2], as views."""
    size = n_pages * kv * PAGE * hd
    return (region[:size].view(n_pages, kv, PAGE, hd), region[size:2 * size].view(n_pages, kv, hd, PAGE),
            region[2 * size:].view(torch.int32).view(n_pages, kv, 2))


def _slots(tables, cached, new):
    """The slot of every new token, sequence by sequence."""
    out = [np.zeros(0, np.int64)]
    for s in range(len(new)):
        p = np.arange(cached[s], cached[s] + new[s])
        out.append(tables[s, p // PAGE].astype(np.int64) * PAGE + p % PAGE)
    return np.concatenate(out)


def prepare(case, seed):
    g, r, kind = _generator(seed), np.random.default_rng(seed + 5), case["kind"]
    if kind == "score":
        return _prepare_score(case, g)
    cached, new = _lengths(case)
    s = {"case": case}
    if kind == "plan":
        held = -(-cached // PAGE) + r.integers(0, 2, len(cached))   # some hold a page more than they use
        width = int((-(-(cached + new) // PAGE)).max()) + 2
        need = np.maximum(-(-(cached + new) // PAGE) - held, 0)
        tables, n_pages, free = _tables(held, width, r, int(need.sum()) + 40)
        s.update(seq_lens=_i32(cached), new_lens=_i32(new), held=_i32(held), free=_i32(free), head=_i32([7]), tables=_i32(tables),
                 max_rows=int(new.sum()) + 5)   # room for a few rows more, as a fixed buffer has
        return s
    dt = DTYPES[case["dtype"]]
    kv, hd = case["kv"], case["hd"]
    total = cached + new
    held = -(-total // PAGE)
    tables, n_pages, _ = _tables(held, int(held.max()) + 1, r)
    s.update(region=_region(n_pages, kv, hd, g), n_pages=n_pages, kv=kv, hd=hd, dt=dt)
    if kind == "append":
        rows = int(new.sum())
        # the rows as a fused projection leaves them: keys and values side by side, some channels much larger
        x = torch.empty(rows, 2, kv, hd, device="cuda").normal_(0.0, 1.0, generator=g)
        x[:, 0, :, 3::29] *= 9.0
        x = x.to(dt)
        s.update(k=x[:, 0], v=x[:, 1], slots=torch.from_numpy(_slots(tables, cached, new)).to("cuda"))
        first = cached // PAGE * PAGE     # the live tokens of the touched pages
        s["check"] = torch.from_numpy(_slots(tables, first, total - first)).to("cuda")
        if own:
            from paper_2606_03113_amd import lede
            s["cache"] = lede.Cache(n_pages, kv, hd, region=s["region"])
        return s
    rows = int(new.sum())
    q = torch.empty(rows, case["q"], hd, device="cuda").normal_(0.0, 1.0, generator=g).to(dt)
    s.update(q=q, tables=_i32(tables), kv_lens=_i32(total), row_start=_i32(np.concatenate([[0], np.cumsum(new)])),
             lens=[int(x) for x in total], new=[int(x) for x in new], max_new=int(new.max()), max_kv=int(total.max()))
    if own:
        from paper_2606_03113_amd import lede
        s["cache"] = lede.Cache(n_pages, kv, hd, region=s["region"])
    return s


def _prepare_score(case, g):
    rows, V = case["rows"], case["vocab"]
    z = torch.empty(rows, V, device="cuda").normal_(0.0, 2.5, generator=g)
    peak = torch.randint(0, V, (rows,), device="cuda", generator=g)
    z[torch.arange(rows, device="cuda"), peak] += 9.0
    banned = torch.rand(rows, V, device="cuda", generator=g) < 0.05      # every other row: a grammar's mask
    banned[1::2] = False
    z = z.masked_fill_(banned, float("-inf")).to(DTYPES[case["dtype"]])
    tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.5, peak, torch.randint(0, V, (rows,), device="cuda", generator=g))
    return {"case": case, "logits": z, "tokens": tokens.to(torch.int32)}


# ---- the operators in elementary operations ------------------------------------------------


def _plain_plan(s):
    seq, new, held = s["seq_lens"].long(), s["new_lens"].long(), s["held"].long()
    tables, n = s["tables"], s["seq_lens"].numel()
    total = seq + new
    need = torch.clamp((total + PAGE - 1) // PAGE - held, min=0)
    head = s["head"].long()
    first = head + torch.cumsum(need, 0) - need
    col = torch.arange(tables.shape[1], device="cuda")
    took = (col >= held[:, None]) & (col < (held + need)[:, None])
    src = torch.where(took, first[:, None] + col - held[:, None], 0)
    tables.copy_(torch.where(took, s["free"][src], tables))
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(new, 0)])
    r = torch.arange(s["max_rows"], device="cuda")
    seq_of = torch.clamp(torch.searchsorted(row_start, r, right=True) - 1, max=n - 1)
    pos = seq[seq_of] + r - row_start[seq_of]
    live = r < row_start[-1]
    page = tables[seq_of, torch.where(live, pos // PAGE, 0)].long()
    slots = torch.where(live, page * PAGE + pos % PAGE, -1)
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    status = torch.cat([zero, row_start[-1:], head + need.sum(), zero - 1])
    return total.int(), (held + need).int(), row_start.int(), slots, tables, status.int()


def _exponent(amax):
    """The smallest e >= E_MIN with amax <= 448 * 2**e."""
    m, x = torch.frexp(amax)                  # amax = m * 2**x, m in [0.5, 1): 448 = 0.875 * 2**9
    e = torch.where(m > 0.875, x - 8, x - 9)
    return torch.clamp(torch.where(amax > 0, e, E_MIN), min=E_MIN)


def _decode(codes, exponent):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), exponent)


def _encode(x):
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    kc, vc, words = _parts(s["region"], s["n_pages"], s["kv"], s["hd"])
    page, off = s["slots"] // PAGE, s["slots"] % PAGE
    pages, local = torch.unique(page, return_inverse=True)
    P = pages.numel()
    mine = torch.zeros(P, PAGE, dtype=torch.bool, device="cuda")
    mine[local, off] = True
    for which, rows, codes in ((0, s["k"], kc), (1, s["v"], vc)):
        x = rows.float()                                                       # [rows][head][dim]
        old = codes[pages] if which == 0 else codes[pages].transpose(2, 3)     # [P][head][64][dim]
        new = torch.zeros(P, PAGE, s["kv"], s["hd"], device="cuda")
        new[local, off] = x
        new = new.transpose(1, 2)
        finite = torch.isfinite(new)
        e_new = _exponent(torch.where(finite, new.abs(), 0.0).amax((2, 3)))
        word = words[pages, :, which]
        fresh = mine[:, 0][:, None]
        e_old = torch.clamp((word & 255) - 127, min=E_MIN)
        e = torch.where(fresh, e_new, torch.maximum(e_old, e_new))
        moved = _encode(torch.ldexp(old.contiguous().view(torch.float8_e4m3fn).float(), (e_old - e)[:, :, None, None]))
        kept = torch.where(fresh[:, :, None, None], old, moved)
        mixed = torch.where(mine[:, None, :, None], _encode(torch.ldexp(new, -e[:, :, None, None])), kept)
        codes[pages] = mixed if which == 0 else mixed.transpose(2, 3)
        bad = (~finite).any(3).any(2) | (((word & NAN_BIT) != 0) & ~fresh)
        words[pages, :, which] = (e + 127 + NAN_BIT * bad).int()
    page, off = s["check"] // PAGE, s["check"] % PAGE
    e = ((words[page] & 255) - 127)[..., None]
    return _decode(kc[page, :, off], e[:, :, 0]).to(s["dt"]), _decode(vc[page, :, :, off], e[:, :, 1]).to(s["dt"])


def _plain_attend(s):
    case, kv, hd = s["case"], s["kv"], s["hd"]
    kc, vc, words = _parts(s["region"], s["n_pages"], kv, hd)
    group = case["q"] // kv
    out = torch.zeros(s["q"].shape, dtype=s["dt"], device="cuda")
    row = 0
    for i, (length, n) in enumerate(zip(s["lens"], s["new"])):
        if n == 0:
            continue
        pages = s["tables"][i, :-(-length // PAGE)].long()
        e = ((words[pages] & 255) - 127)[..., None, None]
        k = _decode(kc[pages], e[:, :, 0]).permute(1, 3, 0, 2).reshape(kv, hd, -1)[:, :, :length].contiguous()
        v = _decode(vc[pages], e[:, :, 1]).permute(1, 0, 3, 2).reshape(kv, -1, hd)[:, :length].contiguous()
        q = s["q"][row:row + n].float().view(n, kv, group, hd).permute(1, 0, 2, 3).reshape(kv, n * group, hd)
        z = torch.matmul(q, k) * hd ** -0.5
        pos = length - n + torch.arange(n, device="cuda")
        seen = torch.arange(length, device="cuda") <= pos[:, None].expand(n, group).reshape(-1, 1)
        z = torch.where(seen, z, float("-inf"))
        p = torch.exp(z - z.amax(-1, keepdim=True))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        out[row:row + n] = o.view(kv, n, group, hd).permute(1, 0, 2, 3).reshape(n, case["q"], hd).to(s["dt"])
        row += n
    return out


def _plain_score(s):
    case, tokens = s["case"], s["tokens"].long()
    rows, V, top = case["rows"], case["vocab"], case["top"]
    parts = []
    index = torch.arange(V, device="cuda")
    for r0 in range(0, rows, 256):
        raw = s["logits"][r0:r0 + 256].float() + 0.0
        tok = tokens[r0:r0 + 256, None]
        z = raw / case["temperature"]
        m = z.amax(1, keepdim=True)
        d = z - m
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        log_total = torch.log(total)
        entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
        own_z = raw.gather(1, tok)
        rank = ((raw > own_z) | ((raw == own_z) & (index < tok))).sum(1)
        bits = raw.view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32 | (0xFFFFFFFF - index)
        ids = 0xFFFFFFFF - (torch.topk(key, top, dim=1).values & 0xFFFFFFFF)
        lp = d - log_total
        parts.append((lp.gather(1, tok)[:, 0], rank.int(), entropy[:, 0], ids.int(), lp.gather(1, ids)))
    return tuple(torch.cat(x) for x in zip(*parts))


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "score": _plain_score}[kind](s)
    from paper_2606_03113_amd import lede
    if kind == "plan":
        p = lede.op_cache_plan(s["seq_lens"], s["new_lens"], s["held"], s["free"], s["head"], s["tables"], s["max_rows"])
        return p.kv_lens, p.held, p.row_start, p.slots, s["tables"], p.status
    if kind == "append":
        lede.op_cache_append(s["cache"], s["k"], s["v"], s["slots"])
        return lede.op_cache_read(s["cache"], s["check"], s["dt"])
    if kind == "attend":
        return lede.op_cache_attention(s["cache"], s["q"], s["tables"], s["kv_lens"], s["row_start"], s["max_new"], s["max_kv"])
    r = lede.op_logprobs(s["logits"], s["tokens"], s["case"]["top"], s["case"]["temperature"])
    return r.logprobs, r.ranks, r.entropy, r.top_ids, r.top_logprobs


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "score":
        rows, V, top = case["rows"], case["vocab"], case["top"]
        es = 4 if case["dtype"] == "f32" else 2
        return {"bytes": rows * V * es + rows * (16 + 8 * top), "flops": 6 * rows * V}
    cached, new = _lengths(case)
    n, rows = case["seqs"], int(new.sum())
    if kind == "plan":
        taken = int(np.maximum(-(-(cached + new) // PAGE) + cached // -PAGE, 0).sum())
        return {"bytes": 12 * n + 8 * taken + 12 * n + 4 + 8 * rows + 24, "flops": 4 * (n + rows)}
    es = 4 if case["dtype"] == "f32" else 2
    wide = case["kv"] * case["hd"]
    total = cached + new
    if kind == "append":
        back = int((total - cached // PAGE * PAGE).sum())
        # rows in and their codes out; the touched pages' codes in and values out
        return {"bytes": 2 * wide * (rows * (es + 1) + back * (1 + es)) + 16 * rows + 8 * back, "flops": 4 * wide * rows}
    pairs = int(sum(m * (t - m) + m * (m + 1) // 2 for t, m in zip(total.tolist(), new.tolist())))
    live = int(total[new > 0].sum())
    return {"bytes": 2 * wide * live + 2 * rows * case["q"] * case["hd"] * es, "flops": 4 * case["q"] * case["hd"] * pairs}


# ---- the operators from their definitions, in 64 bits ------------------------------------------


_E4M3 = np.array([math.nan if c & 127 == 127 else
                  (-1.0 if c & 128 else 1.0) * (math.ldexp(8 + (c & 7), (c >> 3 & 15) - 10) if c & 120 else math.ldexp(c & 7, -9))
                  for c in range(256)])


def _exact_plan(s):
    seq, new, held = (s[k].cpu().numpy() for k in ("seq_lens", "new_lens", "held"))
    tables, free, head = s["tables"].cpu().numpy().copy(), s["free"].cpu().numpy(), int(s["head"][0])
    kv, got, start, slots = [], [], [0], []
    for i in range(len(seq)):
        end, have = int(seq[i] + new[i]), int(held[i])
        while have * PAGE < end:
            tables[i, have] = free[head]
            have, head = have + 1, head + 1
        kv.append(end)
        got.append(have)
        start.append(start[-1] + int(new[i]))
        slots += [int(tables[i, p // PAGE]) * PAGE + p % PAGE for p in range(int(seq[i]), end)]
    rows = len(slots)
    slots += [-1] * (s["max_rows"] - rows)
    i32 = lambda a: np.asarray(a, np.int32)  # noqa: E731
    return i32(kv), i32(got), i32(start), np.asarray(slots, np.int64), tables, i32([0, rows, head, -1])


def _nearest_code(x):
    """The e4m3 values nearest to x (|x| <= 448), ties to the even code."""
    a = np.abs(x)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-30))), -6) - 3)
    return np.sign(x) * np.rint(a / step) * step


def _exact_append(s):
    n_pages, kv, hd = s["n_pages"], s["kv"], s["hd"]
    kc, vc, words = (t.cpu().numpy() for t in _parts(s["region"], n_pages, kv, hd))
    slots, check = s["slots"].cpu().numpy(), s["check"].cpu().numpy()
    outs = []
    for which, rows in ((0, s["k"]), (1, s["v"])):
        x = rows.double().cpu().numpy()
        page_of = slots // PAGE
        pages = {}
        for page in np.unique(page_of):
            old = _E4M3[kc[page] if which == 0 else vc[page].transpose(0, 2, 1)].copy()     # [head][64][dim]
            at = np.nonzero(page_of == page)[0]
            new = x[at].transpose(1, 0, 2)                                                  # [head][rows][dim]
            amax = np.abs(new).max((1, 2))
            e = np.maximum(np.ceil(np.log2(np.maximum(amax, 1e-300) / 448.0)), E_MIN)
            e = np.where(amax > 448.0 * np.exp2(e), e + 1, np.where(amax <= 448.0 * np.exp2(e - 1), np.maximum(e - 1, E_MIN), e))
            if not (slots[at] % PAGE == 0).any():
                before = (words[page, :, which] & 255) - 127.0
                e = np.maximum(e, before)
                old = _nearest_code(old * np.exp2(before - e)[:, None, None])
            old[:, slots[at] % PAGE] = _nearest_code(new * np.exp2(-e)[:, None, None])
            pages[int(page)] = old * np.exp2(e)[:, None, None]
        out = np.empty((len(check), kv, hd))
        for i, c in enumerate(check):
            out[i] = pages[int(c) // PAGE][:, int(c) % PAGE]
        outs.append(out)
    return tuple(outs)


def _exact_attend(s):
    case, kv, hd = s["case"], s["kv"], s["hd"]
    kc, vc, words = _parts(s["region"], s["n_pages"], kv, hd)
    value = torch.from_numpy(_E4M3).to("cuda")
    size = torch.exp2((words & 255).double() - 127)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, row = case["q"] // kv, 0
    for i in range(case["seqs"]):
        length, n = s["lens"][i], s["new"][i]
        pages = s["tables"][i, :(length + PAGE - 1) // PAGE].long()
        for h in range(kv if n else 0):
            k = (value[kc[pages, h].long()] * size[pages, h, 0, None, None]).reshape(-1, hd)[:length]
            v = (value[vc[pages, h].long()] * size[pages, h, 1, None, None]).transpose(1, 2).reshape(-1, hd)[:length].contiguous()
            kt = k.t().contiguous()
            for j in range(h * group, (h + 1) * group):
                z = torch.mm(s["q"][row:row + n, j].double(), kt) / math.sqrt(hd)
                z.masked_fill_(torch.ones(n, length, dtype=torch.bool, device="cuda").triu(length - n + 1), -math.inf)
                out[row:row + n, j] = torch.mm(torch.softmax(z, 1), v)
        row += n
    return out


def _exact_score(s):
    case = s["case"]
    outs = []
    for r in range(0, case["rows"], 64):
        raw = s["logits"][r:r + 64].double()
        tok = s["tokens"][r:r + 64].long()[:, None]
        lp = torch.log_softmax(raw / case["temperature"], 1)
        p = torch.exp(lp)
        entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices
        rank = (order == tok).int().argmax(1)
        ids = order[:, :case["top"]]
        outs.append((lp.gather(1, tok)[:, 0], rank.int(), entropy, ids.int(), lp.gather(1, ids)))
    return tuple(torch.cat(x) for x in zip(*outs))


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "attend": _exact_attend, "score": _exact_score}[case["kind"]](s)
