"""The batch operators on the GPU against their plain fp64 counterparts: page plans, appends to and reads from the 8-bit
cache, attention over it, scores of tokens, and a run of them together."""
import math

import numpy as np
import pytest

from tests import batch_reference as ref
from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def lede():
    from paper_2606_03113_amd import lede as m
    return m


def gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    return t if dtype is None else t.to(dtype)


def i32(a):
    return gpu(np.asarray(a, np.int32))


def rounded(a, dtype):
    """The rows as the GPU gets them, and their values."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[dtype])
    return t.to("cuda"), t.double().numpy()


# ---- plans -------------------------------------------------------------------------------------


def _plan_case(r, n, new_hi, cached_hi, extra=0):
    seq = r.integers(0, cached_hi + 1, n)
    new = r.integers(0, new_hi + 1, n)
    held = -(-seq // 64) + r.integers(0, extra + 1, n)
    width = int(max(held.max(), (-(-(seq + new) // 64)).max(), 1)) + 1
    need = int(np.maximum(-(-(seq + new) // 64) - held, 0).sum())
    n_pages = int(held.sum()) + need + 3
    order = r.permutation(n_pages).astype(np.int32)
    tables, at = np.full((n, width), -7, np.int32), 0
    for s in range(n):
        tables[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    return seq, new, held, tables, order[at:], need


def _check_plan(p, tables, want):
    kv, held, start, slots, tab, status = want
    assert p.status.tolist() == status
    assert p.kv_lens.tolist() == kv.tolist() and p.held.tolist() == held.tolist() and p.row_start.tolist() == start.tolist()
    assert np.array_equal(p.slots.cpu().numpy(), slots)
    assert np.array_equal(tables.cpu().numpy(), tab)


@pytest.mark.parametrize("n,new_hi,cached_hi,extra", [(1, 1, 0, 0), (1, 5, 63, 0), (3, 1, 64, 1), (64, 1, 300, 0), (1023, 3, 200, 2),
                                                     (1024, 1, 64, 0), (1025, 2, 130, 1), (2500, 70, 90, 0), (5, 3000, 1000, 1), (2, 0, 10, 0)])
def test_plan(n, new_hi, cached_hi, extra):
    say("plan n=%d new<=%d cached<=%d" % (n, new_hi, cached_hi))
    r = np.random.default_rng(n + new_hi)
    seq, new, held, tables, free, need = _plan_case(r, n, new_hi, cached_hi, extra)
    rows = int(new.sum())
    for max_rows in (rows, rows + 77):
        t = gpu(tables)
        p = lede().op_cache_plan(i32(seq), i32(new), i32(held), i32(free), i32([2]), t, max_rows)
        _check_plan(p, t, ref.plan(seq, new, held, len(free), 2, tables.shape[1], max_rows, free, tables))


def test_plan_failures_take_nothing():
    m = lede()
    r = np.random.default_rng(3)
    seq, new, held, tables, free, need = _plan_case(r, 1400, 40, 100)
    rows = int(new.sum())
    bad = []
    for at in (0, 700, 1399):
        for change in ((seq, -1), (new, -3), (held, -1), (held, tables.shape[1] + 1), (new, 64 * tables.shape[1] + 1), (seq, 1 << 30)):
            bad.append((at, change))
    for at, (field, value) in bad:
        say("plan failure", at, value)
        keep = field[at]
        field[at] = value
        t = gpu(tables)
        p = m.op_cache_plan(i32(seq), i32(new), i32(held), i32(free), i32([0]), t, rows + 100)
        want = ref.plan(seq, new, held, len(free), 0, tables.shape[1], rows + 100, free, tables)
        assert want[-1][0] != 0
        _check_plan(p, t, want)
        field[at] = keep
    for head, n_free, max_rows in ((0, need - 1, rows), (4, len(free), rows), (-1, len(free), rows), (len(free) + 1, len(free), rows), (0, len(free), rows - 1)):
        say("plan pool", head, n_free, max_rows)
        t = gpu(tables)
        p = m.op_cache_plan(i32(seq), i32(new), i32(held), i32(free[:n_free]), i32([head]), t, max_rows)
        want = ref.plan(seq, new, held, n_free, head, tables.shape[1], max_rows, free, tables)
        assert want[-1][0] != 0
        _check_plan(p, t, want)


def test_plan_in_place():
    """Lengths, held pages and the free list's place updated where they are, step after step, with a rollback between."""
    m = lede()
    seq, new, held, free = np.zeros(3, int), np.array([60, 3, 70]), np.zeros(3, int), np.arange(20)[::-1].astype(np.int32)
    tables = np.full((3, 6), -1, np.int32)
    d_seq, d_held, d_tab = i32(seq), i32(held), gpu(tables)
    status = i32([0, 0, 0, -1])
    out = m.CachePlan(d_seq, d_held, torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(200, dtype=torch.int64, device="cuda"), status)
    head = 0
    for step in range(6):
        p = m.op_cache_plan(d_seq, i32(new), d_held, gpu(free), status[2:3], d_tab, 200, out=out)
        want = ref.plan(seq, new, held, len(free), head, 6, 200, free, tables)
        _check_plan(p, d_tab, want)
        seq, held, tables, head = want[0], want[1], want[4], want[5][2]
        if step == 2:   # a rollback keeps the pages
            seq = seq - np.array([4, 0, 60])
            d_seq.copy_(i32(seq))
        new = np.array([1, 40, 5]) + step


# ---- appends and reads -----------------------------------------------------------------------------


def _check_read(cache, model, slots, dtype):
    k, v = lede().op_cache_read(cache, gpu(np.asarray(slots, np.int64)), DT[dtype])
    for got, want in zip((k, v), model.read(slots)):
        # every code's value has 4 significant bits: it is the dtype's own
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


def _rows(r, n, kv, hd, size=1.0):
    x = r.standard_normal((n, 2, kv, hd)) * size
    x[:, 0, :, ::13] *= 20
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kv,hd", [(1, 64), (3, 128), (8, 128), (5, 64)])
def test_append_and_read(dtype, kv, hd):
    """Pages filled in runs of every kind: whole, from the start, inside, to the end, one token, over a page's end; rows
    whose size grows (the page's codes are rounded anew) and shrinks; rows that go nowhere."""
    m = lede()
    say("append", dtype, kv, hd)
    r = np.random.default_rng(kv * hd)
    n_pages = 9
    cache, model = m.Cache(n_pages, kv, hd), ref.CacheModel(n_pages, kv, hd)
    runs = [[(3, 0, 64)], [(5, 0, 10), (1, 0, 1)], [(5, 10, 11), (1, 1, 30), (7, 0, 64), (0, 0, 7)], [(5, 11, 64), (2, 0, 40)], [(1, 30, 31)],
            [(2, 40, 41), (1, 31, 32), (0, 7, 12)], [(3, 5, 9)], [(3, 0, 3)], [(8, 63, 64), (6, 1, 3)]]
    everything = np.arange(n_pages * 64)
    for step, run in enumerate(runs):
        slots = np.concatenate([p * 64 + np.arange(a, b) for p, a, b in run])
        slots = np.concatenate([[-1], slots, [n_pages * 64, -64, 1 << 40]])
        x = _rows(r, len(slots), kv, hd, 2.0 ** [0, 3, -2, 5, 5, 0, 9, -6, 1][step])
        d, val = rounded(x, dtype)
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
        model.append(val[:, 0], val[:, 1], slots)
        _check_read(cache, model, everything, dtype)
    words = cache.region[2 * n_pages * kv * 64 * hd:].view(torch.int32).view(n_pages, kv, 2).cpu().numpy()
    touched = [0, 1, 2, 3, 5, 6, 7, 8]
    assert np.array_equal(words[touched] - 127, model.e.transpose(1, 2, 0)[touched])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_values(dtype):
    """Every rounding of e4m3 at several scales, zeros, the smallest and the largest values, and what is not finite."""
    m = lede()
    cache, model = m.Cache(8, 2, 64), ref.CacheModel(8, 2, 64)
    x = np.zeros((8 * 64, 2, 2, 64), np.float32)
    grid = np.ldexp(np.arange(-480, 481), -14).astype(np.float32)
    x[:64, 0, 0] = np.resize(grid * 2048, (64, 64))
    x[64:128, 0, 0] = np.resize(np.concatenate([grid, [448.0]]), (64, 64))
    x[128:192, 0, 1] = 448.0
    x[192:256, 0, 1, 5] = 448.01 if dtype == "f32" else 450.0
    x[256:320, 1, 0] = np.resize(np.float32([1e-38, 1e-45, -1e-30, 2.0 ** -110, 2.0 ** -109, 2.0 ** -92]), (64, 64))
    x[320:384, 1, 0, 0] = 3.0e38
    x[384:448, 0, 0, 7] = np.inf
    x[400, 1, 1, 9], x[401, 0, 1, 3] = np.nan, -np.inf
    x[384:448, 0, 0, 8] = np.linspace(-3, 3, 64)
    d, val = rounded(x, dtype)
    slots = np.arange(512)
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
    model.append(val[:, 0], val[:, 1], slots)
    _check_read(cache, model, slots, dtype)


@pytest.mark.parametrize("kv,rows", [(2, 5000), (40, 700), (1, 1)])
def test_append_many_rows(kv, rows):
    """Windows of one row and of many; runs over window borders; strided rows of a wider buffer."""
    m = lede()
    say("append rows=%d" % rows)
    r = np.random.default_rng(rows)
    n_pages, hd = 97, 64
    cache, model = m.Cache(n_pages, kv, hd), ref.CacheModel(n_pages, kv, hd)
    pages = r.permutation(n_pages)
    slots, left = [], rows
    for p in pages:
        a = int(r.integers(0, 64))
        b = int(r.integers(a + 1, 65)) if r.random() < 0.5 else 64
        slots.append(p * 64 + np.arange(a, b)[:left])
        left -= len(slots[-1])
        if left <= 0:
            break
    slots = np.concatenate(slots)
    x = _rows(r, len(slots), kv, hd)
    d, val = rounded(x, "bf16")
    wide = torch.zeros(len(slots), 3 * kv * hd + 8, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 2 * kv * hd] = d.view(len(slots), -1)
    k, v = (wide[:, 8 + i * kv * hd:8 + (i + 1) * kv * hd].unflatten(1, (kv, hd)) for i in (0, 1))
    m.op_cache_append(cache, k, v, gpu(slots))
    model.append(val[:, 0], val[:, 1], slots)
    _check_read(cache, model, np.arange(n_pages * 64), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_read_any_order_and_untouched_rows(dtype, hd):
    m = lede()
    r = np.random.default_rng(hd)
    kv, n_pages = 3, 11
    cache, model = m.Cache(n_pages, kv, hd), ref.CacheModel(n_pages, kv, hd)
    slots = np.arange(n_pages * 64)
    d, val = rounded(_rows(r, len(slots), kv, hd), dtype)
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
    model.append(val[:, 0], val[:, 1], slots)
    for n in (1, 7, 300, 1000):
        want = r.integers(0, n_pages * 64, n)      # some twice
        want[n // 2:] = np.sort(want[n // 2:])
        _check_read(cache, model, want, dtype)
        out = torch.full((2, n, kv + 1, hd), 7.0, dtype=DT[dtype], device="cuda")[:, :, :kv]
        given = want.copy()
        given[::3] = [-1, n_pages * 64, -(1 << 50)][n % 3]
        m.op_cache_read(cache, gpu(given), DT[dtype], out=(out[0], out[1]))
        left = torch.ones(n, dtype=torch.bool)
        left[::3] = False
        for got, ok in zip(out, model.read(want)):
            got = got.double().cpu().numpy()
            assert (got[::3] == 7.0).all() and np.array_equal(got[left.numpy()], ok[left.numpy()])


# ---- attention ----------------------------------------------------------------------------------------


def _fill(kv, hd, lens, r, dtype="bf16", spare=2, size=1.0, poison=True):
    """A cache with sequences of the given lengths on pages in random order; unwritten places hold NaN codes."""
    m = lede()
    held = [-(-n // 64) for n in lens]
    n_pages = sum(held) + spare
    cache, model = m.Cache(n_pages, kv, hd), ref.CacheModel(n_pages, kv, hd)
    if poison:
        cache.region[:2 * n_pages * kv * 64 * hd] = 0x7F
    order, at = r.permutation(n_pages), 0
    tables = np.full((len(lens), max(held + [1]) + 1), -1, np.int32)
    for s, n in enumerate(lens):
        tables[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
        if n:
            p = np.arange(n)
            slots = tables[s, p // 64].astype(np.int64) * 64 + p % 64
            d, val = rounded(_rows(r, n, kv, hd, size), dtype)
            m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
            model.append(val[:, 0], val[:, 1], slots)
    return cache, model, tables


def _attend(cache, model, tables, lens, new, nq, dtype, r, max_new=None, max_kv=None, scale=None, q=None):
    m = lede()
    start = np.concatenate([[0], np.cumsum(new)])
    rows = int(start[-1])
    d, val = rounded(r.standard_normal((rows + 2, nq, cache.head_dim)) if q is None else q, dtype)
    out = torch.full((rows + 2, nq, cache.head_dim), 5.0, dtype=DT[dtype], device="cuda")
    got = m.op_cache_attention(cache, d, gpu(tables), i32(lens), i32(start), max(new) if max_new is None else max_new,
                               max(lens) if max_kv is None else max_kv, scale=scale, out=out).double().cpu().numpy()
    want, tol = ref.attention(model, val, tables, lens, start, cache.head_dim ** -0.5 if scale is None else scale, dtype)
    assert (got[rows:] == 5.0).all()
    got, want, tol = got[:rows], want[:rows], tol[:rows]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert not np.isnan(tol[ok]).any()
    over = np.abs(got - want)[ok] - tol[ok]
    assert over.size == 0 or over.max() <= 0, "over the tolerance by %.3g (of %.3g)" % (over.max(), tol[ok][over.argmax()])
    return got


HEADS = [(4, 4, 64), (8, 2, 128), (32, 8, 128), (7, 1, 64), (28, 4, 128), (5, 5, 128), (40, 1, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,kv,hd", HEADS)
def test_attention_ragged(dtype, nq, kv, hd):
    """Lengths around page ends, nothing new, nothing cached, more rows than tokens (the first see nothing)."""
    say("attention", dtype, nq, kv, hd)
    r = np.random.default_rng(nq * hd)
    lens = [1, 63, 64, 65, 0, 0, 128, 200, 3, 131, 5]
    new = [1, 1, 1, 2, 0, 3, 0, 5, 3, 17, 9]
    cache, model, tables = _fill(kv, hd, lens, r)
    _attend(cache, model, tables, lens, new, nq, dtype, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,kv,hd,length,new", [(4, 2, 64, 3000, 1), (16, 2, 128, 2049, 5), (6, 6, 128, 1025, 1), (9, 1, 64, 1500, 33), (8, 1, 128, 700, 129)])
def test_attention_long(dtype, nq, kv, hd, length, new):
    """Long axes, split over blocks and joined; one sequence, and beside short ones."""
    say("attention long", dtype, nq, kv, hd, length, new)
    r = np.random.default_rng(length)
    lens, news = [length, 40, 257], [new, 1, 2]
    cache, model, tables = _fill(kv, hd, lens, r)
    _attend(cache, model, tables, lens, news, nq, dtype, r)
    _attend(cache, model, tables[:1], lens[:1], news[:1], nq, dtype, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_expected_sizes_only_spread_the_work(dtype):
    r = np.random.default_rng(8)
    lens, new = [900, 70, 333], [20, 1, 333]
    cache, model, tables = _fill(2, 64, lens, r)
    for max_new, max_kv in ((0, 0), (1, 1), (1, 100000), (5000, 64), (20, 900), (2 ** 20, 2 ** 20)):
        say("attention sizes", max_new, max_kv)
        _attend(cache, model, tables, lens, new, 6, dtype, r, max_new=max_new, max_kv=max_kv)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("expect", [None, 600])   # rows expected: the variant for few, and the one for many
def test_attention_peaked_flat_and_scaled(dtype, expect):
    """Scores that one token dominates, equal scores, huge ones, other scales (a negative one, zero)."""
    r = np.random.default_rng(9)
    lens, new = [300, 65], [3, 2]
    cache, model, tables = _fill(2, 64, lens, r)
    for scale, size in ((1.0, 3.0), (0.0, 1.0), (-0.2, 1.0), (0.125, 1e-20), (1e-3, 100.0)):
        say("attention scale", scale, size)
        q = r.standard_normal((7, 4, 64)) * size
        _attend(cache, model, tables, lens, new, 4, dtype, r, scale=scale, q=q, max_new=expect)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("expect", [None, 600])   # rows expected: the variant for few, and the one for many
def test_attention_many_small_weights(dtype, rows, expect):
    """One token with most of the weight, and thousands whose weights are below fp16's normal range beside it."""
    m = lede()
    r = np.random.default_rng(rows)
    kv, hd, length = 1, 64, 6000
    cache, model = m.Cache(length // 64 + 1, kv, hd), ref.CacheModel(length // 64 + 1, kv, hd)
    for gap in (12, 17, 20, 24):      # nats below the first token: e^-17 = 2^-24.5
        x = np.zeros((length, 2, kv, hd))
        x[:, 0, :, 0] = -gap
        x[:rows, 0, :, 0] = 0.0       # (every row sees one)
        x[:, 1] = 1.0 + r.random((length, kv, hd))
        d, val = rounded(x, "bf16")
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
        model = ref.CacheModel(length // 64 + 1, kv, hd)
        model.append(val[:, 0], val[:, 1], np.arange(length))
        q = np.zeros((rows + 2, 2, hd))
        q[:, :, 0] = 1.0
        _attend(cache, model, np.arange(length // 64 + 1, dtype=np.int32)[None], [length], [rows], 2, dtype, r, scale=1.0, q=q, max_new=expect)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [2, 70])
@pytest.mark.parametrize("expect", [None, 600])   # rows expected: the variant for few, and the one for many
def test_attention_huge_scores(dtype, rows, expect):
    """Scores far beyond fp32's whole numbers: the largest one's value, to the output's rounding."""
    m = lede()
    kv, hd, length = 1, 64, 300
    r = np.random.default_rng(rows)
    cache, model = m.Cache(5, kv, hd), ref.CacheModel(5, kv, hd)
    x = np.zeros((length, 2, kv, hd))
    x[:, 0, 0, 0] = 1.0 + np.arange(length) % 7 / 8        # distinct sizes; the largest is one token's
    best = 150
    x[best, 0, 0, 0] = 4.0
    x[:, 1] = r.standard_normal((length, kv, hd)) * np.exp2(np.arange(length) // 64 * 3)[:, None, None]   # blocks of several scales
    d, val = rounded(x, "bf16")
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(np.arange(length)))
    model.append(val[:, 0], val[:, 1], np.arange(length))
    value = model.read([best])[1][0, 0]
    table = np.arange(5, dtype=np.int32)[None]
    for size in (3e3, 1e6, 3e7, 1e8, 3e8, 1e9, 1e11, 1e20, 1e30):
        q = np.zeros((rows, 1, hd), np.float32)
        q[:, 0, 0] = size
        got = m.op_cache_attention(cache, rounded(q, dtype)[0], gpu(table), i32([length]), i32([0, rows]), expect or rows, length, scale=1.0)
        got = got.double().cpu().numpy()
        assert (np.abs(got - value) <= ref.HALF_STEP[dtype] * 2 * np.abs(value)).all(), size
        # the other way, the largest scores are the most negative ones' opposites
        got = m.op_cache_attention(cache, rounded(-q, dtype)[0], gpu(table), i32([length]), i32([0, rows]), expect or rows, length, scale=-1.0)
        assert (np.abs(got.double().cpu().numpy() - value) <= ref.HALF_STEP[dtype] * 2 * np.abs(value)).all(), size


@pytest.mark.parametrize("dtype,seqs,nq,kv,new,hd", [("bf16", 131, 4, 4, 1, 64), ("f32", 200, 3, 3, 2, 64), ("bf16", 9, 60, 60, 70, 64), ("bf16", 70, 8, 8, 9, 64),
                                                     ("f32", 70, 8, 8, 17, 64), ("bf16", 3, 60, 60, 400, 64), ("bf16", 3, 80, 40, 300, 64), ("bf16", 3, 60, 60, 400, 128),
                                                     ("f32", 3, 32, 16, 400, 128), ("bf16", 70, 48, 8, 8, 128)])
def test_attention_more_tasks_than_a_round(dtype, seqs, nq, kv, new, hd):
    """Whole rounds of blocks and a cut rest, few and many rows."""
    say("attention tasks", dtype, seqs, nq, kv, new)
    r = np.random.default_rng(seqs)
    lens = [int(x) for x in r.integers(new, new + (900 if seqs < 10 else 400), seqs)]
    news = [int(x) for x in r.integers(max(1, new - 3), new + 1, seqs)]
    cache, model, tables = _fill(kv, hd, lens, r)
    m = lede()
    cut = [m.load().lede_op_cache_attention_bytes(int(dtype == "bf16"), seqs, sum(news), nq, kv, hd, max(news), n) > 0 for n in (max(lens), 40000)]
    assert cut[1] or (kv, new, hd) == (60, 400, 64)       # (where contexts may be long, but for thousands of tasks)
    start = np.concatenate([[0], np.cumsum(news)])
    d, val = rounded(r.standard_normal((int(start[-1]), nq, hd)), dtype)
    both = [m.op_cache_attention(cache, d, gpu(tables), i32(lens), i32(start), max(news), n).double().cpu().numpy() for n in (max(lens), 40000)]
    for s in np.unique(np.concatenate([[0, seqs - 1], r.integers(0, seqs, 12)])):     # some of them: the reference takes its time
        rows = np.unique(np.concatenate([[start[s], start[s + 1] - 1], r.integers(start[s], start[s + 1], 6)]))
        heads = np.unique(r.integers(0, nq, 5))
        k, v = model.sequence(tables[s], lens[s])
        for row in rows:
            seen = lens[s] - (start[s + 1] - row) + 1
            for h in heads:
                z = hd ** -0.5 * (k[:seen, h // (nq // kv)] @ val[row, h])
                w = np.exp(z - z.max())
                w /= w.sum()
                want = w @ v[:seen, h // (nq // kv)]
                eps = 2.0 ** -23 * (200 * 0.125 * (np.abs(k[:seen, h // (nq // kv)]) @ np.abs(val[row, h])).max() + 200) + (2.0 ** -12 if dtype == "bf16" else 2.0 ** -22)
                tol = 2 * eps * (w @ np.abs(v[:seen, h // (nq // kv)])) + ref.HALF_STEP[dtype] * np.abs(want) * (1 + 2 ** -6)
                for got in both:
                    assert (np.abs(got[row, h] - want) <= tol).all(), (s, row, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,kv,hd", HEADS)
@pytest.mark.parametrize("rows", [16, 64])
def test_attention_many_short_sequences(dtype, nq, kv, hd, rows):
    """More tasks than a round of short contexts, most of them with nothing to do; rows above the expected number, an
    infinite value that some rows see, a page outside the pool, output in place."""
    m, most = lede(), rows // (nq // kv)
    say("attention short", dtype, nq, kv, hd)
    r = np.random.default_rng(nq + hd)
    none = [0] * (600 // kv)
    lens, new = [1, 63, 64, 65, 0, 0, 128, 450, 3, 131, 5] + none, [1, 1, 1, 2, 0, 3, 0, 5, 3, 17, 9] + none
    cache, model, tables = _fill(kv, hd, lens, r)
    assert rows > 16 or m.load().lede_op_cache_attention_bytes(int(dtype == "bf16"), len(lens), sum(new), nq, kv, hd, most, 450) == 0
    _attend(cache, model, tables, lens, new, nq, dtype, r, max_new=most)
    slot = np.array([tables[9, 120 // 64].astype(np.int64) * 64 + 120 % 64])       # rows of the tenth sequence end at 130
    x = _rows(r, 1, kv, hd)
    x[0, 1, kv - 1, 17] = np.inf
    d, val = rounded(x, dtype)
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slot))
    model.append(val[:, 0], val[:, 1], slot)
    got = _attend(cache, model, tables, lens, new, nq, dtype, r, max_new=most)
    assert 0 < np.isnan(got).sum() < got.size / 3
    start = np.concatenate([[0], np.cumsum(new)])
    q, _ = rounded(r.standard_normal((int(start[-1]), nq, hd)), dtype)
    tables[7, 7] = cache.n_pages       # tokens 448 ..: its last two rows
    args = (gpu(tables), i32(lens), i32(start), most, 450)
    out = m.op_cache_attention(cache, q, *args)
    end = int(start[8])
    assert torch.isnan(out[end - 2:end]).all() and not torch.isnan(out[end - 5:end - 2]).any()
    assert torch.equal(torch.nan_to_num(m.op_cache_attention(cache, q, *args, out=q), 7.0), torch.nan_to_num(out, 7.0))


def test_attention_one_long_sequence_among_short_ones():
    """Contexts of which one is far longer: its pages are spread over many blocks, the others are whole."""
    r = np.random.default_rng(21)
    lens, new = [20000, 64, 700, 1, 129], [1, 1, 1, 1, 1]
    cache, model, tables = _fill(2, 64, lens, r)
    for dtype in ("bf16", "f32"):
        _attend(cache, model, tables, lens, new, 4, dtype, r)


def test_attention_blocks_of_different_scale():
    """Pages whose values differ by 2^60: a row that attends to the small one alone sees its own precision."""
    m = lede()
    r = np.random.default_rng(10)
    kv, hd = 1, 64
    cache, model = m.Cache(3, kv, hd), ref.CacheModel(3, kv, hd)
    for page, ks, vs in ((2, 0.0, 2.0 ** 30), (0, 40.0, 2.0 ** -30), (1, 0.0, 1.0)):
        x = np.stack([np.full((64, kv, hd), ks / hd), r.standard_normal((64, kv, hd)) * vs], 1)
        d, val = rounded(x, "bf16")
        slots = page * 64 + np.arange(64)
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
        model.append(val[:, 0], val[:, 1], slots)
    tables = np.array([[2, 0, 1]], np.int32)
    for dtype in ("f32", "bf16"):
        for expect in (1, 20, 600):
            _attend(cache, model, tables, [192], [1], 2, dtype, r, scale=1.0, q=np.full((3, 2, hd), 2.0), max_new=expect)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [6, 40])
@pytest.mark.parametrize("expect", [None, 600])   # rows expected: the variant for few, and the one for many
def test_attention_nan_stays_with_the_rows_that_see_it(dtype, rows, expect):
    """NaN and infinite keys and values at positions that some rows of a pass see and earlier ones do not; a query row
    that is not finite."""
    m = lede()
    say("attention nan", dtype, rows)
    r = np.random.default_rng(rows)
    kv, hd, length = 2, 64, 250
    for where in ("k", "v"):
        cache, model, tables = _fill(kv, hd, [length, 70], r)
        pos = np.array([length - rows + 3])
        slots = tables[0, pos // 64].astype(np.int64) * 64 + pos % 64
        x = _rows(r, 1, kv, hd)
        x[0, 0 if where == "k" else 1, 1, 17] = np.nan if rows == 6 else np.inf
        d, val = rounded(x, dtype)
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(slots))
        model.append(val[:, 0], val[:, 1], slots)
        got = _attend(cache, model, tables, [length, 70], [rows, 2], 6, dtype, r, max_new=expect)
        assert np.isnan(got[3:rows, 3:]).any() and not np.isnan(got[:3]).any() and not np.isnan(got[:, :3]).any() and not np.isnan(got[rows:]).any()
    cache, model, tables = _fill(kv, hd, [length, 70], r)
    q = r.standard_normal((rows + 4, 6, hd))
    q[2, 4, 5] = np.nan
    got = _attend(cache, model, tables, [length, 70], [rows, 2], 6, dtype, r, q=q, max_new=expect)
    assert np.isnan(got[2, 4]).all() and np.isnan(got).sum() == hd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 70])
@pytest.mark.parametrize("expect", [None, 600])   # rows expected: the variant for few, and the one for many
def test_attention_pages_outside_the_pool(dtype, rows, expect):
    """An entry of a table that names no page: rows that see it are NaN, others are right; entries that no row sees may be
    anything.  Lengths above the table's and row starts outside the rows are held to them."""
    m = lede()
    r = np.random.default_rng(rows)
    kv, hd, lens = 2, 128, [200, 130]
    for bad in (-1, 1 << 30, -(2 ** 31)):
        say("attention page", bad)
        cache, model, tables = _fill(kv, hd, lens, r)
        bad = cache.n_pages if bad == 1 << 30 else bad
        tables[0, 3] = bad            # tokens 192 ..
        new = [rows, 2]
        start = np.array([0, rows, rows + 2])
        d, val = rounded(r.standard_normal((rows + 2, 4, hd)), dtype)
        got = m.op_cache_attention(cache, d, gpu(tables), i32(lens), i32(start), expect or rows, 200).double().cpu().numpy()
        sees = np.concatenate([200 - rows + np.arange(rows) >= 192, [False, False]])
        assert np.isnan(got[sees]).all() and not np.isnan(got[~sees]).any()
        good = tables.copy()
        good[0, 3] = good[0, 2]
        want, tol = ref.attention(model, val, good, lens, start, hd ** -0.5, dtype)
        assert (np.abs(got - want)[~sees] <= tol[~sees]).all()
    # too long for its table: as many tokens as the table holds
    cache, model, tables = _fill(kv, hd, lens, r)
    short = tables[:, :3].copy()
    d, val = rounded(r.standard_normal((3, 4, hd)), dtype)
    got = m.op_cache_attention(cache, d, gpu(short), i32([200, 130]), i32([-5, 1, 2]), expect or 1, 200).double().cpu().numpy()
    want, tol = ref.attention(model, val, short, [192, 130], [0, 1, 2], hd ** -0.5, dtype)
    assert (np.abs(got - want)[:2] <= tol[:2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_strides_and_workspace(dtype):
    m = lede()
    r = np.random.default_rng(12)
    lens, new = [1300, 90], [2, 1]
    cache, model, tables = _fill(2, 64, lens, r)
    d, val = rounded(r.standard_normal((3, 4, 64)), dtype)
    want, tol = ref.attention(model, val, tables, lens, [0, 2, 3], 0.125, dtype)
    wide = torch.full((3, 6 * 64 + 8), 3.0, dtype=DT[dtype], device="cuda")
    wide[:, 8:8 + 256] = d.view(3, -1)
    out = torch.full((3, 5 * 64), 3.0, dtype=DT[dtype], device="cuda")
    need = m.load().lede_op_cache_attention_bytes(int(dtype == "bf16"), 2, 3, 4, 2, 64, 2, 1300)
    assert need > 0
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        m.op_cache_attention(cache, wide[:, 8:8 + 256].unflatten(1, (4, 64)), gpu(tables), i32(lens), i32([0, 2, 3]), 2, 1300,
                             out=out[:, :256].unflatten(1, (4, 64)), workspace=ws[:need])
        got = out[:, :256].unflatten(1, (4, 64)).double().cpu().numpy()
        assert (np.abs(got - want) <= tol).all() and (out[:, 256:] == 3.0).all() and (ws[need:] == 0xFF).all()
    with pytest.raises(m.LedeError):
        m.op_cache_attention(cache, d, gpu(tables), i32(lens), i32([0, 2, 3]), 2, 1300, workspace=ws[:need - 16])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [[1, 0, 2], [9, 1, 3], [20, 2, 1], [70, 0, 1], [200, 1, 3]])
def test_attention_in_place(dtype, new):
    """The output in the queries' own rows, beside splits that are joined later: the bits of an output of its own."""
    m = lede()
    say("in place", dtype, new)
    r = np.random.default_rng(sum(new))
    lens = [900, 70, 2000]
    cache, model, tables = _fill(2, 64, lens, r)
    start = i32(np.concatenate([[0], np.cumsum(new)]))
    q, _ = rounded(r.standard_normal((sum(new) + 1, 6, 64)), dtype)
    args = (gpu(tables), i32(lens), start, max(new), max(lens))
    want = torch.full_like(q, 3.0)
    want[-1] = q[-1]
    m.op_cache_attention(cache, q, *args, out=want)
    assert m.op_cache_attention(cache, q, *args, out=q) is q
    assert torch.equal(q, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [[1, 1, 1], [30, 2, 5], [66, 4, 1], [130, 4, 1]])
def test_attention_shared_pages(dtype, new):
    """Requests with one beginning read the same pages; a page may even stand twice in one table."""
    r = np.random.default_rng(19)
    lens = [190, 250, 130]
    cache, model, tables = _fill(3, 128, lens, r)
    tables[1, :2] = tables[0, :2]
    tables[2, 1] = tables[2, 0]
    _attend(cache, model, tables, lens, new, 6, dtype, r)


def test_attention_page_started_anew():
    """A page that held NaNs and large values, given to another request: nothing of them stays."""
    m = lede()
    r = np.random.default_rng(20)
    cache, model, tables = _fill(2, 64, [70], r, size=1e4)
    bad = torch.full((3, 2, 64), math.nan, device="cuda")
    slots = tables[0, 0].astype(np.int64) * 64 + np.arange(3)
    m.op_cache_append(cache, bad, bad, gpu(slots + 20))
    for dtype, rows, expect in (("f32", 2, None), ("bf16", 40, None), ("bf16", 40, 600)):
        d, val = rounded(_rows(r, 45, 2, 64, 1e-3), dtype)
        at = tables[0, 0].astype(np.int64) * 64 + np.arange(45)
        m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(at))
        model.append(val[:, 0], val[:, 1], at)
        got = _attend(cache, model, tables, [45], [rows], 4, dtype, r, max_new=expect)
        assert np.isfinite(got).all() and np.abs(got).max() < 1e-2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("expect", [4, 8, 600])
def test_attention_rows_do_not_depend_on_the_batch(dtype, expect):
    """The same bits again, and with other lengths, rows and queries beside."""
    m = lede()
    r = np.random.default_rng(13)
    lens, new = [2000, 500, 77], [1, 4, 1]
    cache, model, tables = _fill(4, 128, lens, r)
    d, _ = rounded(r.standard_normal((6, 16, 128)), dtype)
    args = (gpu(tables), i32(lens), i32([0, 1, 5, 6]), expect, 2000)
    a, b = m.op_cache_attention(cache, d, *args), m.op_cache_attention(cache, d, *args)
    assert torch.equal(a, b)
    e = torch.cat([d[:1], 30 * d[1:3], d[5:]])
    c = m.op_cache_attention(cache, e, gpu(tables), i32([2000, 130, 77]), i32([0, 1, 3, 4]), expect, 2000)
    assert torch.equal(c[0], a[0]) and torch.equal(c[3], a[5]) and not torch.equal(c[1], a[1])


# ---- scores ----------------------------------------------------------------------------------------------


def _score(z, tokens, top, T, dtype, pitch=0, shift=0):
    m = lede()
    rows, V = z.shape
    t = torch.from_numpy(np.ascontiguousarray(z, dtype=np.float32)).to(DT[dtype])
    wide = torch.full((rows, V + pitch + shift), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, shift:shift + V] = t.to("cuda")
    got = m.op_logprobs(wide[:, shift:shift + V], None if tokens is None else i32(tokens), top, T)
    for r in range(rows):
        lp, rank, h, ids, tlp = ref.scores(t[r].double().numpy(), T, -1 if tokens is None else int(tokens[r]), top)

        def close(a, b):
            a = np.asarray(a.cpu(), np.float64)
            b = np.asarray(b, np.float64)
            same = (a == b) | (np.isnan(a) & np.isnan(b))
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(a - b) <= ref.score_tolerance(b, V))).all(), (r, a, b)
        close(got.entropy[r], h)
        if tokens is not None:
            close(got.logprobs[r], lp)
            assert int(got.ranks[r]) == rank, r
        assert got.top_ids[r].tolist() == list(ids), r
        close(got.top_logprobs[r], tlp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (3, 2, 2), (2, 33, 32), (5, 1000, 5), (1, 8192, 32), (2, 8193, 20), (3, 8191, 1), (2, 16390, 32),
                                       (4, 50257, 20), (1, 128256, 32), (7, 97, 0)])
def test_logprobs(dtype, rows, V, top):
    say("logprobs", dtype, rows, V, top)
    r = np.random.default_rng(V)
    z = r.standard_normal((rows, V)) * 3
    tokens = r.integers(0, V, rows)
    tokens[0] = z[0].argmax()
    _score(z, tokens, top, 1.0, dtype)
    _score(z, tokens, top, 0.6, dtype, pitch=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 3, 5, 7])
def test_logprobs_any_alignment(dtype, shift):
    r = np.random.default_rng(shift)
    for V in (8185, 16384):
        z = r.standard_normal((3, V)) * 2
        z[:, 0] = 9.0            # the first and the last entries count
        z[:, -1] = 8.0
        _score(z, [0, V - 1, 5], 4, 1.3, dtype, pitch=shift, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_ties_masks_and_what_is_not_finite(dtype):
    V = 9000
    r = np.random.default_rng(4)
    inf, nan = np.inf, np.nan
    z = r.standard_normal((14, V))
    z[0] = 2.5                                  # all equal
    z[1] = r.integers(0, 3, V)                  # many ties
    z[2, :] = -inf
    z[2, [17, 8500]] = [1.0, 0.0]               # two tokens left
    z[3] = -inf                                 # none left
    z[4, 100] = nan
    z[5, [4, 8999]] = nan
    z[6, 77] = inf
    z[7, [3, 5]] = [inf, nan]
    z[8, ::2] = 0.0
    z[8, 1::2] = -0.0                           # zeros of both signs are equal
    z[9] = np.finfo(np.float32).min * (0.9 if dtype == "f32" else 0.5)
    z[10, 50] = 200.0                           # one token is certain
    z[11] = -inf
    z[11, 8999] = -3.0
    z[12] = nan
    z[13, :8192] = -inf                         # a whole segment masked
    tokens = [4000, 7, 8500, 5, 100, 8999, 77, 3, 6001, 0, 51, 8999, 8990, 1]
    _score(z, tokens, 32, 1.0, dtype)
    _score(z, [V, -1, 17, -5, 99, 5, 5, 5, 0, 8999, 50, 0, 0, 8200], 3, 0.7, dtype)
    _score(z[:, :200], None, 20, 1.0, dtype)


def test_logprobs_largest_vocabulary():
    """The most entries and top tokens that are taken: rows of random logits, of equal ones, and with a mask of all but a few."""
    V = 1 << 20
    r = np.random.default_rng(6)
    z = r.standard_normal((3, V))
    z[1] = -1.25
    z[2] = -np.inf
    z[2, [5, 70000, V - 1]] = [1.0, 2.0, 1.0]
    _score(z, [V - 1, 12345, 70000], 32, 1.0, "bf16")
    _score(z, [0, V - 1, 5], 7, 0.8, "f32")


def test_logprobs_rising_rows():
    """Logits that rise or fall along the row: every tile holds larger ones than those before."""
    V = 30000
    z = np.stack([np.linspace(-5, 5, V), np.linspace(5, -5, V), np.sin(np.arange(V) / 300.0), np.floor(np.linspace(0, 40, V))])
    for dtype in ("f32", "bf16"):
        _score(z, [V - 1, V - 1, 471, 100], 32, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("each", [1, 17, 31, 32, 40])
def test_logprobs_equal_tops_in_every_part(dtype, each):
    """As many largest entries, equal or nearly, in every part of a long row: none of the parts has the row's top tokens."""
    V = 1 << 20
    r = np.random.default_rng(each)
    z = -1.0 - r.random((2, V))
    at = (np.arange(0, V - 8192, 8192)[:, None] + 100 + 3 * np.arange(each)).reshape(-1)
    z[0, at] = 5.0
    z[1, at] = 5.0 + r.integers(0, 2, len(at)) / 32
    _score(z, [at[-1], 0], 32, 1.0, dtype)


@pytest.mark.parametrize("rows,V", [(1100, 40001), (530, 135001)])
def test_logprobs_many_rows(rows, V):
    """More rows than a round of blocks, a row a block and with rows cut in parts (few rows, or longer than a block takes): each against the same row alone."""
    m = lede()
    r = np.random.default_rng(7)
    z = gpu(r.standard_normal((rows, V)).astype(np.float32) * 2)
    tok = i32(r.integers(0, V, rows))
    all_rows, few = m.op_logprobs(z, tok, 9, 0.7), m.op_logprobs(z[300:340], tok[300:340], 9, 0.7)
    for a, b in ((all_rows.ranks, few.ranks), (all_rows.top_ids, few.top_ids)):
        assert torch.equal(a[300:340], b)
    lp = torch.log_softmax(z.double() / 0.7, 1)
    want = lp.gather(1, tok.long()[:, None])[:, 0]
    tol = ref.score_tolerance(want.cpu().numpy(), V)
    assert (np.abs(all_rows.logprobs.double().cpu().numpy() - want.cpu().numpy()) <= tol).all()
    ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :9]
    assert torch.equal(all_rows.top_ids.long(), ids)


def test_logprobs_extreme_temperatures_and_logits():
    r = np.random.default_rng(5)
    z = r.standard_normal((3, 700)) * 40
    for T in (0.01, 1e-3, 50.0, 1e6):
        say("logprobs T", T)
        _score(z, [1, 2, int(z[2].argmax())], 3, T, "f32")


# ---- together -----------------------------------------------------------------------------------------------


class Batch:
    """A one-layer decoder of random weights over the operators: K/V of a token are rows of a table, queries another's,
    the head a linear product."""

    def __init__(self, seed, seqs, nq=8, kv=2, hd=64, vocab=304, dtype="bf16", pages=24, width=6):
        m = lede()
        r = np.random.default_rng(seed)
        self.nq, self.kv, self.hd, self.vocab, self.dtype, self.seqs = nq, kv, hd, vocab, dtype, seqs
        self.qkv, self.qkv_val = rounded(r.standard_normal((vocab, nq + 2 * kv, hd)), dtype)
        self.head, self.head_val = rounded(r.standard_normal((vocab, nq * hd)) * 0.2, dtype)
        self.cache, self.model = m.Cache(pages, kv, hd), ref.CacheModel(pages, kv, hd)
        self.free_val = r.permutation(pages).astype(np.int32)
        self.free = gpu(self.free_val)
        self.tables = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
        self.lens, self.held = i32(np.zeros(seqs)), i32(np.zeros(seqs))
        self.status = i32([0, 0, 0, -1])
        self.start = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
        self.tiled = torch.empty(m.load().lede_op_tiled_bytes(1, vocab, nq * hd), dtype=torch.uint8, device="cuda")
        assert m.load().lede_op_repack(1, self.head.data_ptr(), vocab, nq * hd, self.tiled.data_ptr(), self.stream()) == 0

    @staticmethod
    def stream():
        return torch.cuda.current_stream().cuda_stream

    def buffers(self, rows):
        m = lede()
        return m.CachePlan(self.lens, self.held, self.start, torch.empty(rows, dtype=torch.int64, device="cuda"), self.status)

    def step(self, new, tokens, targets, plan, out, logits, max_new):
        """One pass of tokens [rows <= 16]: plan, append, attention, head, scores."""
        m = lede()
        m.op_cache_plan(self.lens, new, self.held, self.free, self.status[2:3], self.tables, plan.slots.numel(), out=plan)
        x = self.qkv[tokens]
        m.op_cache_append(self.cache, x[:, self.nq:self.nq + self.kv], x[:, self.nq + self.kv:], plan.slots)
        m.op_cache_attention(self.cache, x[:, :self.nq], self.tables, plan.kv_lens, plan.row_start, max_new, 64 * self.tables.shape[1], out=out)
        rows = tokens.numel()
        assert m.load().lede_op_linear(1, self.tiled.data_ptr(), self.vocab, self.nq * self.hd, out.data_ptr(), self.nq * self.hd, rows,
                                       logits.data_ptr(), 1, self.stream()) == 0
        return m.op_logprobs(logits, targets, 4)


def test_batch_run():
    """Prompts, decoding steps, a rollback and a further pass of ragged requests, every operator's result against its
    counterpart on what the operator before it gave."""
    b = Batch(1, 3)
    r = np.random.default_rng(2)
    lens, held, tables, head = np.zeros(3, int), np.zeros(3, int), np.full((3, 6), -1, np.int32), 0
    for step, new in enumerate([[5, 1, 9], [1, 1, 1], [0, 7, 2], [4, 4, 4], [1, 0, 15]] + [[1, 1, 1]] * 3 + [[5, 6, 5]] * 8):
        rows, pad = sum(new), 2 if sum(new) < 15 else 0
        tokens, targets = r.integers(0, b.vocab, rows + pad), r.integers(0, b.vocab, rows + pad)
        plan = b.buffers(rows + pad)
        out = torch.zeros(rows + pad, b.nq, b.hd, dtype=torch.bfloat16, device="cuda")
        logits = torch.zeros(rows + pad, b.vocab, device="cuda")
        got = b.step(i32(new), gpu(tokens), i32(targets), plan, out, logits, max(new))
        want = ref.plan(lens, new, held, len(b.free_val), head, 6, rows + pad, b.free_val, tables)
        _check_plan(plan, b.tables, want)
        lens, held, tables, head = want[0], want[1], want[4], want[5][2]
        x = b.qkv_val[tokens]
        b.model.append(x[:, b.nq:b.nq + b.kv], x[:, b.nq + b.kv:], want[3])
        o, tol = ref.attention(b.model, x[:, :b.nq], tables, lens, want[2], 0.125, "bf16")
        assert (np.abs(out.double().cpu().numpy() - o)[:rows] <= tol[:rows]).all()
        y = out.double().cpu().numpy().reshape(rows + pad, -1)
        z = y @ b.head_val.T
        size = np.abs(y) @ np.abs(b.head_val).T
        zz = logits.double().cpu().numpy()
        assert (np.abs(zz - z) <= 2.0 ** -23 * (b.nq * b.hd) * size + 1e-30).all()
        for i in range(rows):
            lp, rank, h, ids, tlp = ref.scores(zz[i], 1.0, int(targets[i]), 4)
            assert int(got.ranks[i]) == rank and got.top_ids[i].tolist() == list(ids)
            assert abs(float(got.logprobs[i]) - lp) <= ref.score_tolerance(lp, b.vocab)
            assert abs(float(got.entropy[i]) - h) <= ref.score_tolerance(h, b.vocab)
        if step == 3:       # drafts rejected: the tokens leave, their pages stay
            lens = lens - np.array([3, 0, 2])
            b.lens.copy_(i32(lens))


def test_batch_run_in_a_graph():
    """A captured decoding step, replayed: lengths, pages and the free list advance on the device alone."""
    eager, b = Batch(5, 4), Batch(5, 4)
    new = i32([1, 1, 0, 3])
    steps = np.random.default_rng(6).integers(0, eager.vocab, (90, 2, 5))

    def make(x):
        plan = x.buffers(7)     # a padded pass: five rows of seven
        return plan, torch.zeros(7, x.nq, x.hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(7, x.vocab, device="cuda")

    tokens, targets = torch.zeros(7, dtype=torch.int64, device="cuda"), torch.zeros(7, dtype=torch.int32, device="cuda")
    plan, out, logits = make(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        res = b.step(new, tokens, targets, plan, out, logits, 3)
    e_plan, e_out, e_logits = make(eager)
    for i, (tok, tar) in enumerate(steps):
        tokens[:5], targets[:5] = gpu(tok), i32(tar)
        want = eager.step(new, tokens, targets, e_plan, e_out, e_logits, 3)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((plan.kv_lens, e_plan.kv_lens), (plan.held, e_plan.held), (plan.slots, e_plan.slots), (plan.status, e_plan.status),
                     (b.tables, eager.tables), (out, e_out), (res.logprobs[:5], want.logprobs[:5]), (res.ranks[:5], want.ranks[:5]),
                     (res.top_ids[:5], want.top_ids[:5]), (res.entropy[:5], want.entropy[:5])):
            assert torch.equal(x, y), i
        assert int(plan.status[0]) == 0


def test_on_another_stream():
    """Work on a stream of its own, ordered by its events alone."""
    m = lede()
    r = np.random.default_rng(14)
    lens, new = [1500, 200], [1, 3]
    cache, model, tables = _fill(2, 128, lens, r)
    d, val = rounded(r.standard_normal((4, 8, 128)), "bf16")
    z, tok = gpu(r.standard_normal((4, 5000)).astype(np.float32)), i32([1, 2, 3, 4])
    args = (gpu(tables), i32(lens), i32([0, 1, 4]), 3, 1500)
    a, b = m.op_cache_attention(cache, d, *args), m.op_logprobs(z, tok, 8, 0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c, e = m.op_cache_attention(cache, d, *args), m.op_logprobs(z, tok, 8, 0.9)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, c) and torch.equal(b.logprobs, e.logprobs) and torch.equal(b.top_ids, e.top_ids)


def test_two_streams_at_once():
    """Calls that overlap on two streams, each with a workspace and outputs of its own."""
    m = lede()
    r = np.random.default_rng(21)
    lens, new = [6000, 40, 300, 2500], [2, 1, 1, 1]
    cache, model, tables = _fill(2, 64, lens, r)
    q = [rounded(r.standard_normal((5, 8, 64)), "bf16")[0] for _ in range(2)]
    z = [gpu(r.standard_normal((5, 60000)).astype(np.float32)) for _ in range(2)]
    args = (gpu(tables), i32(lens), i32([0, 2, 3, 4, 5]), 2, 6000)
    tok = i32([1, 2, 3, 4, 59999])
    want = [(m.op_cache_attention(cache, q[i], *args), m.op_logprobs(z[i], tok, 32)) for i in range(2)]
    need = m.load().lede_op_cache_attention_bytes(1, 4, 5, 8, 2, 64, 2, 6000), m.load().lede_op_logprobs_bytes(5, 60000, 32)
    assert min(need) > 0
    ws = [[torch.empty(n, dtype=torch.uint8, device="cuda") for n in need] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append((m.op_cache_attention(cache, q[i], *args, workspace=ws[i][0]), m.op_logprobs(z[i], tok, 32, workspace=ws[i][1])))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lp in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lp.top_ids, want[i][1].top_ids)
            assert torch.equal(lp.logprobs, want[i][1].logprobs) and torch.equal(lp.entropy, want[i][1].entropy)


def test_long_cache_offsets():
    """A cache of more than 4 GiB of codes: pages at its end."""
    m = lede()
    kv, hd = 8, 128
    n_pages = (1 << 32) // (kv * 64 * hd) + 40
    say("cache of %.1f GiB" % (2 * n_pages * kv * 64 * hd / 2 ** 30))
    cache = m.Cache(n_pages, kv, hd)
    r = np.random.default_rng(15)
    pages = np.array([n_pages - 1, 0, n_pages - 17])
    small = ref.CacheModel(3, kv, hd)
    length = 150
    p = np.arange(length)
    d, val = rounded(_rows(r, length, kv, hd), "bf16")
    m.op_cache_append(cache, d[:, 0], d[:, 1], gpu(pages[p // 64].astype(np.int64) * 64 + p % 64))
    small.append(val[:, 0], val[:, 1], p)
    k, v = m.op_cache_read(cache, gpu(pages[p // 64].astype(np.int64) * 64 + p % 64), torch.float32)
    wk, wv = small.read(p)
    assert np.array_equal(k.double().cpu().numpy(), wk) and np.array_equal(v.double().cpu().numpy(), wv)
    q, qv = rounded(r.standard_normal((2, 16, hd)), "bf16")
    got = m.op_cache_attention(cache, q, i32(pages[None]), i32([length]), i32([0, 2]), 2, length).double().cpu().numpy()
    want, tol = ref.attention(small, qv, np.array([[0, 1, 2]]), [length], [0, 2], hd ** -0.5, "bf16")
    assert (np.abs(got - want) <= tol).all()
    assert math.isfinite(got.sum())
