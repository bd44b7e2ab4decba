"""The batch operators where magnitudes are far apart, against their plain fp64 counterparts: pages whose values differ by
many powers of two, in every variant of the attention, and scores of logits far from zero or of low temperatures."""
import numpy as np
import pytest

from tests import batch_reference as ref
from tests.parity import say
from tests.test_gpu_batch_ops import _attend, _fill, gpu, lede, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# (sequences, rows and cached tokens expected), which choose the variant and how pages are split; the work itself is
# that of a few rows behind some pages
VARIANTS = {
    "rows16": (2, 1, 40000),          # a block's waves take every fourth page
    "rows16-cut": (2, 1, 768),        # and a page each, three splits joined
    "alone": (300, 1, 400),           # a wave has all pages
    "rows32": (2, 12, 40000),
    "rows32-cut": (2, 12, 768),
    "rows64": (2, 30, 40000),         # waves take rows, and all of them every page
    "rows64-cut": (2, 30, 768),
    "rows64-more": (300, 30, 768),    # more blocks than a round: pages as codes (bf16)
    "rows128": (2, 2000, 40000),      # (bf16)
    "rows128-more": (60, 1000, 768),
}
KV, NQ = 2, 4


def _check(variant, dtype, hd, sizes, r, keys=None, q=None, values=None, scale=None):
    """One sequence whose pages' values have the given sizes (0: all zero), beside a short one and empty ones."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    length = 64 * len(sizes) - 5
    lens, new = [length, 70] + [0] * (seqs - 2), [3, 1] + [0] * (seqs - 2)
    cache, model, tables = _fill(KV, hd, lens, r)
    x = r.standard_normal((length, 2, KV, hd)) if values is None else values(length)
    x[:, 0] *= 0.3
    if keys is not None:
        x[:, 0] = keys(length)[:, None, None]
    x[:, 1] *= np.repeat(np.asarray(sizes, float), 64)[:length, None, None]
    d, val = rounded(x, "bf16")
    p = np.arange(length)
    slots = tables[0, p // 64].astype(np.int64) * 64 + p % 64
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
    model.append(val[:, 0], val[:, 1], slots)
    return _attend(cache, model, tables, lens, new, NQ, dtype, r, max_new=max_new, max_kv=max_kv, q=q, scale=scale)


def _sizes(pattern, n=12):
    """The sizes of a sequence's pages."""
    if pattern == "zeros-behind":
        return [1.0 if p % 3 == 0 else 0.0 for p in range(n)]
    if pattern == "zeros-before":
        return [0.0 if p < 5 else 1.0 for p in range(n)]
    if pattern == "zero-last":
        return [1.0] * 6 + [0.0] + [1.0] * (n - 7)
    where, ratio = pattern.split("/")
    at = {"first": (0, 1, 2, 3), "middle": (2, 5, 8), "last": (6, n - 1), "one": (1,)}[where]
    small, large = {"20": (-10, 10), "33": (0, 33), "60": (-30, 30), "100": (-60, 40), "190": (-90, 100)}[ratio]
    return [2.0 ** (large if p in at else small) for p in range(n)]


PATTERNS = ["zeros-behind", "zeros-before", "zero-last"] + [w + "/" + x for x in ("20", "33", "60", "100", "190") for w in ("first", "middle", "last", "one")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_pages_of_any_size_keep_their_weight(dtype, hd, variant):
    """A page has its part of the softmax whatever its values are: all zero, or smaller or larger than others' by many
    powers of two, before and behind them."""
    r = np.random.default_rng(hd)
    for pattern in PATTERNS:
        say("attention sizes", dtype, hd, variant, pattern)
        _check(variant, dtype, hd, _sizes(pattern), r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_small_weights_of_small_pages(dtype, hd, variant):
    """Thousands of tokens 12 nats below one whose page has values 2^16 larger hold some percent of the weight."""
    r = np.random.default_rng(31)
    q = np.full((6, NQ, hd), 16.0 / hd)
    for gap in (10.0, 12.0, 13.0):
        say("attention gap", dtype, variant, gap)
        # (q.k = 16 k: the first token's score is `gap` nats larger)
        _check(variant, dtype, hd, [2.0 ** 16] * 4 + [1.0] * 60, r, keys=lambda n: np.where(np.arange(n) == 0, gap / 4, -gap / 4), q=q, scale=0.125)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_scores_as_large_as_fp32_holds(dtype, hd, variant):
    """Scores up to fp32's largest, and ordinary ones of the largest and smallest keys."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    r = np.random.default_rng(55)
    length, best = 300, 150
    lens, start = np.array([length] + [0] * (seqs - 1), np.int32), np.array([0] + [3] * seqs, np.int32)
    table = np.tile(np.arange(5, dtype=np.int32), (seqs, 1))
    cache, model = m.Cache(5, KV, hd), ref.CacheModel(5, KV, hd)
    x = np.zeros((length, 2, KV, hd))
    x[:, 0, :, 0] = (1.0 + np.arange(length) % 7 / 8)[:, None]
    x[best, 0, :, 0] = 2.25
    x[:, 1] = r.standard_normal((length, KV, hd))
    d, val = rounded(x, "bf16")
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
    model.append(val[:, 0], val[:, 1], np.arange(length))
    for size in (1e35, 3e36, 1e37, 1e38):
        say("attention largest", dtype, variant, size)
        q = np.zeros((3, NQ, hd), np.float32)
        q[:, :, 0] = size
        got = m.op_cache_attention(cache, rounded(q, dtype)[0], gpu(table), gpu(lens), gpu(start), max_new, max_kv, scale=1.0)
        got = got.double().cpu().numpy()
        for h in range(NQ):      # (the best token's weight is a power of two: two half steps are the quotient's and the output's)
            want = model.read([best])[1][0, h // (NQ // KV)]
            assert (np.abs(got[:, h] - want) <= ref.HALF_STEP[dtype] * 2 * np.abs(want)).all(), (size, h)
    for k in (-90, 100, 118):
        say("attention keys", dtype, variant, k)
        cache, model = m.Cache(5, KV, hd), ref.CacheModel(5, KV, hd)
        x = r.standard_normal((length, 2, KV, hd))
        x[:, 0] *= 0.3 * 2.0 ** k
        d, val = rounded(x, "bf16")
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
        model.append(val[:, 0], val[:, 1], np.arange(length))
        q = r.standard_normal((5, NQ, hd)) * 2.0 ** -k
        _attend(cache, model, table, lens.tolist(), [3] + [0] * (seqs - 1), NQ, dtype, r, max_new=max_new, max_kv=max_kv, q=q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_hugely_negative_scores(dtype, hd, variant):
    """Rows all of whose scores are far below zero: the largest one's value, as long as fp32 holds the scores."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    r = np.random.default_rng(61)
    kv, length, best = 2, 300, 150
    cache, model = m.Cache(5, kv, hd), ref.CacheModel(5, kv, hd)
    x = np.zeros((length, 2, kv, hd))
    x[:, 0, :, 0] = (1.0 + np.arange(length) % 7 / 8)[:, None]
    x[best, 0, :, 0] = 0.5
    x[:, 1] = r.standard_normal((length, kv, hd)) * np.exp2(np.arange(length) // 64 * 3)[:, None, None]
    d, val = rounded(x, "bf16")
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
    model.append(val[:, 0], val[:, 1], np.arange(length))
    value = model.read([best])[1][0, 0], model.read([best])[1][0, 1]
    # The best token's weight is the sum.  bf16: both are the same 11 bits, so the output's rounding is all, with room for as
    # much again.  fp32: half steps of the weight in two parts (2 x 11 bits, 1), of its two products in the accumulator, whose
    # additions may cut off (2 each), of the reciprocal, of the product with it and of the exponential in the sum (1 each).
    steps = 2 if dtype == "bf16" else 8
    table = np.tile(np.arange(5, dtype=np.int32), (seqs, 1))
    start = np.array([0] + [3] * seqs, np.int32)
    lens = np.array([length] + [0] * (seqs - 1), np.int32)
    for size in (1e3, 1e8, 1e20, 1e29, 1e30, 3e30, 1e32, 1e35, 1e37, 1e38):
        say("attention negative", dtype, variant, size)
        q = np.zeros((3, NQ, hd), np.float32)
        q[:, :, 0] = -size
        got = m.op_cache_attention(cache, rounded(q, dtype)[0], gpu(table), gpu(lens), gpu(start), max_new, max_kv, scale=1.0)
        got = got.double().cpu().numpy()
        for h in range(NQ):
            want = value[h // (NQ // kv)]
            assert (np.abs(got[:, h] - want) <= ref.HALF_STEP[dtype] * steps * np.abs(want)).all(), (size, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_pages_never_written(dtype, hd, variant):
    """Pages of a cleared cache that no append has reached are tokens of zero keys and values."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    r = np.random.default_rng(51)
    n = 7
    length = 64 * n - 9
    for written in ((1, 2, 3, 4, 5, 6), (0, 5), (6,)):
        say("attention cleared", dtype, variant, written)
        cache, model = m.Cache(n + 1, KV, hd), ref.CacheModel(n + 1, KV, hd)
        for page in written:
            d, val = rounded(r.standard_normal((64, 2, KV, hd)), "bf16")
            slots = page * 64 + np.arange(64)
            m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
            model.append(val[:, 0], val[:, 1], slots)
        tables = np.tile(np.arange(n, dtype=np.int32), (seqs, 1))
        _attend(cache, model, tables, [length, 70] + [0] * (seqs - 2), [3, 1] + [0] * (seqs - 2), NQ, dtype, r, max_new=max_new, max_kv=max_kv)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_dims_that_only_small_pages_have(dtype, variant):
    """Large pages whose values are zero but for one dim: the others' sums are the small pages' alone."""
    r = np.random.default_rng(41)
    for ratio in (10, 25, 40, 60):
        for at in ((0,), (3, 4), (0, 2, 5)):
            say("attention dims", dtype, variant, ratio, at)

            def values(n):
                x = r.standard_normal((n, 2, KV, 128))
                x[np.isin(np.arange(n) // 64, at), 1, :, 1:] = 0.0
                return x
            sizes = [2.0 ** (ratio - ratio // 2 if p in at else -(ratio // 2)) for p in range(12)]
            _check(variant, dtype, 128, sizes, r, values=values)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_pages_of_no_weight_beside_small_ones(dtype, hd, variant):
    """Pages all of whose scores fp32 does not hold, -infinity, behind and before pages of small values: no weight, and the
    others keep theirs."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    r = np.random.default_rng(71)
    n = 12
    length = 64 * n
    for far, small in (((2, 5, 8, 9, 10), (1, 4, 7)), ((4, 5, 6, 7), (1, 2, 3)), ((11,), (7, 8, 9, 10)), ((0, 1, 2, 3), (4, 5, 6, 7))):
        say("attention no weight", dtype, variant, far, small)
        x = r.standard_normal((length, 2, KV, hd))
        page = np.arange(length) // 64
        x[:, 0, :, 0] = np.where(np.isin(page, far), 30.0, 0.0)[:, None]      # times q's 1e38: beyond fp32, or nothing
        x[:, 0, :, 1:] *= 0.3
        x[np.isin(page, small), 1] *= 2.0 ** -30
        cache, model = m.Cache(n, KV, hd), ref.CacheModel(n, KV, hd)
        d, val = rounded(x, "bf16")
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
        model.append(val[:, 0], val[:, 1], np.arange(length))
        q = r.standard_normal((6, NQ, hd))
        q[:, :, 0] = -1e38
        start = [0, 4] + [4] * (seqs - 1)
        got = m.op_cache_attention(cache, rounded(q, dtype)[0], gpu(np.tile(np.arange(n, dtype=np.int32), (seqs, 1))), gpu(np.array([length] + [0] * (seqs - 1), np.int32)),
                                   gpu(np.array(start, np.int32)), max_new, max_kv).double().cpu().numpy()[:4]
        # the others' keys have a zero against 1e38
        kk, vv = model.read(np.arange(length))
        qv = rounded(q, dtype)[1][:4]
        for i in range(4):
            seen = ~np.isin(page, far) & (np.arange(length) <= length - 4 + i)
            for h in range(NQ):
                k, v = kk[seen, h // 2, 1:], vv[seen, h // 2]
                z = hd ** -0.5 * (k @ qv[i, h, 1:])
                w = np.exp(z - z.max())
                w /= w.sum()
                want = w @ v
                # (as ref.attention counts)
                terms = (3 * hd + 4) * hd ** -0.5 * (np.abs(k) @ np.abs(qv[i, h, 1:])).max() + 4 + 2 * (80 + n)
                eps = 2.0 ** -23 * terms + (2.0 ** -12 if dtype == "bf16" else 2.0 ** -22)
                tol = 2 * eps * (w @ np.abs(v)) + ref.HALF_STEP[dtype] * np.abs(want) * (1 + 2 ** -6)
                assert (np.abs(got[i, h] - want) <= tol).all(), (i, h)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_attention_largest_fp32_queries(hd, variant):
    """fp32 queries between bf16's largest number and their own."""
    m = lede()
    seqs, max_new, max_kv = VARIANTS[variant]
    r = np.random.default_rng(81)
    length, best = 300, 100
    cache, model = m.Cache(5, KV, hd), ref.CacheModel(5, KV, hd)
    x = r.standard_normal((length, 2, KV, hd))
    x[:, 0] = 0.0
    x[:, 0, :, 0] = 0.25
    x[best, 0, :, 0] = 0.5
    d, val = rounded(x, "bf16")
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
    model.append(val[:, 0], val[:, 1], np.arange(length))
    q = np.zeros((3, NQ, hd), np.float32)
    for size in (3.39e38, 3.3999e38, -3.4e38):
        say("attention queries", hd, variant, size)
        q[:, :, 0] = size
        got = m.op_cache_attention(cache, gpu(q), gpu(np.tile(np.arange(5, dtype=np.int32), (seqs, 1))), gpu(np.array([length] + [0] * (seqs - 1), np.int32)),
                                   gpu(np.array([0] + [3] * seqs, np.int32)), max_new, max_kv, scale=float(np.sign(size))).double().cpu().numpy()
        for h in range(NQ):      # (the best token's weight is a power of two: two half steps are the quotient's and the output's)
            want = model.read([best])[1][0, h // (NQ // KV)]
            assert (np.abs(got[:, h] - want) <= ref.HALF_STEP["f32"] * 2 * np.abs(want)).all(), (size, h)


# ---- scores ----------------------------------------------------------------------------------------------------


def _close(got, z, T, tokens, top):
    for i in range(len(z)):
        lp, rank, h, ids, tlp = ref.scores(z[i], T, -1 if tokens is None else int(tokens[i]), top)
        for a, b in ((got.entropy[i], h), (got.top_logprobs[i], tlp)) + (((got.logprobs[i], lp),) if tokens is not None else ()):
            a, b = np.asarray(a.cpu(), np.float64), np.asarray(b, np.float64)
            assert (np.abs(a - b) <= ref.score_tolerance(b, z.shape[1])).all(), (i, a, b)
        assert tokens is None or int(got.ranks[i]) == rank
        assert got.top_ids[i].tolist() == list(ids)


def _far_rows(r, V, size):
    """Logits whose magnitude is far above their differences, the largest at different places, and equal ones."""
    z = r.standard_normal((5, V)) * 5 * max(1.0, size / 2 ** 22)
    z[1, V // 2] = z[1].max() + 30
    z[2] = 0.0
    z[3, : V - 8192] = -3.0
    return z + np.array([size, size, size, -size, -size])[:, None]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3 * 8192 + 40, 60001])        # whole rows, and rows in parts that are joined
def test_logprobs_temperatures_near_zero(dtype, V):
    """Low temperatures over rows of whole tiles: the largest products of a logit and 1/T, small differences among them."""
    r = np.random.default_rng(V)
    z, val = rounded(np.concatenate([r.standard_normal((2, V)) * 5, r.standard_normal((1, V)) * 1e-5 + 12.0, np.full((1, V), -7.3)]), dtype)
    tokens = np.array([3, int(val[1].argmax()), V - 1, 20000], np.int32)
    for T in (1e-2, 1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 1e-12, 1e-30):
        for given in (tokens, None):
            say("logprobs", dtype, V, T, given is None)
            _close(lede().op_logprobs(z, None if given is None else gpu(given), 8, T), val, T, given, 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3 * 8192 + 40, 60001])
def test_logprobs_far_logits(dtype, V):
    """Logits far from zero, as masks and offsets leave them, over rows of whole tiles."""
    r = np.random.default_rng(V + 1)
    for size in (1e3, 65504.0, 1e6, 1e7, 1e9, 1e20, 1e36):
        z, val = rounded(_far_rows(r, V, size), dtype)
        tokens = np.array([V - 1, 0, 9000, V - 1, 5], np.int32)
        for given in (tokens, None):
            say("logprobs", dtype, V, size, given is None)
            _close(lede().op_logprobs(z, None if given is None else gpu(given), 8), val, 1.0, given, 8)
