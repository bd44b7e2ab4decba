"""The life of the batch cache's pages on the GPU against plain counterparts: forks, pages made a sequence's own, copies,
pages freed, compaction, and a run of them with plans, appends and attention."""
import numpy as np
import pytest

from tests import batch_reference as ref
from tests.pages_reference import PAGE, Pool, pages
from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def lede():
    from paper_2606_03113_amd import lede as m
    return m


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to("cuda")


class Device:
    """The GPU's copy of a pool; guards behind every array stay as they were."""

    def __init__(self, pool):
        self.parts, self.guards = {}, {}
        for name, a in (("seq", pool.seq), ("held", pool.held), ("tables", pool.tables), ("shares", pool.shares()), ("free", pool.free)):
            flat = i32(np.concatenate([np.asarray(a).reshape(-1), np.full(70, 12345)]))
            n = np.asarray(a).size
            self.parts[name], self.guards[name] = flat[:n].view(np.asarray(a).shape), flat[n:]
        self.status = i32([0, 0, pool.head, -1])
        self.head = self.status[2:3]

    def __getattr__(self, name):
        return self.parts[name]

    def check(self, pool, status=None, pairs=None, got=None):
        for name, want in (("seq", pool.seq), ("held", pool.held), ("shares", pool.shares())):
            assert np.array_equal(self.parts[name].cpu().numpy(), want), name
        got_tab = self.tables.cpu().numpy()
        assert np.array_equal(got_tab, pool.tables)
        assert np.array_equal(self.free.cpu().numpy(), pool.free)
        for name, g in self.guards.items():
            assert bool((g == 12345).all()), name
        if got is not None:
            assert got.status.tolist() == status
            g = got.pairs.cpu().numpy()
            assert [tuple(p) for p in g[:len(pairs)]] == pairs and (g[len(pairs):] == -1).all()


def _pool(r, n, ctx, extra=0, spare=8, empty=0.0, width=None):
    """Sequences of up to ctx tokens, some holding more pages than they need, some none."""
    seq = r.integers(0, ctx + 1, n)
    held = -(-seq // PAGE) + r.integers(0, extra + 1, n)
    gone = r.random(n) < empty
    seq[gone] = held[gone] = 0
    width = max(int(held.max()), 1) + 2 if width is None else width
    n_pages = int(held.sum()) + spare
    order, tables, at = r.permutation(n_pages), np.full((n, width), -7), 0
    for s in range(n):
        tables[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    return Pool(seq, held, tables, order, at, n_pages)


def _forks(r, pool, share=0.7, prefix=0.3):
    """Forks into the empty sequences of the pool."""
    n = len(pool.seq)
    source, lens = np.full(n, -1), r.integers(-5, 500, n)      # (lens of what is no fork are not read)
    parents = np.nonzero(pool.held > 0)[0]
    for s in np.nonzero(pool.held == 0)[0]:
        if len(parents) and r.random() < share:
            source[s] = r.choice(parents)
            lens[s] = r.integers(0, pool.seq[source[s]] + 1) if r.random() < prefix else pool.seq[source[s]]
    return source, lens


@pytest.mark.parametrize("n,ctx", [(2, 1), (2, 64), (9, 200), (64, 3000), (1023, 70), (1025, 130), (2100, 65), (3, 20000)])
def test_fork_and_own(n, ctx):
    m = lede()
    for seed in range(3):
        say("fork n=%d ctx=%d seed=%d" % (n, ctx, seed))
        r = np.random.default_rng(seed * 1000 + n)
        pool = _pool(r, n, ctx, extra=2, spare=3 * n + 8, empty=0.5)
        d = Device(pool)
        source, lens = _forks(r, pool)
        whole = seed == 2
        want = pool.fork(source, None if whole else lens)
        got = m.op_cache_fork(i32(source), d.seq, d.held, d.tables, d.shares, lens=None if whole else i32(lens))
        assert want[0] == 0 and got.tolist() == want
        d.check(pool)
        new = r.integers(0, 3, n) if seed else r.integers(0, 300, n)
        for _ in range(2):     # the second time there is nothing left to do
            max_moves = n
            status, pairs = pool.own(new, max_moves)
            assert status[0] == 0
            got = m.op_cache_own(d.seq, i32(new), d.held, d.free, d.head, d.tables, d.shares, max_moves, out=m.CacheMoves(
                torch.empty(max_moves, 2, dtype=torch.int32, device="cuda"), d.status))
            d.check(pool, status, pairs, got)
        assert not pairs


def test_all_holders_write():
    """Of a page that all of its holders write the first sequence keeps it; a holder that does not write keeps it for itself."""
    m = lede()
    for writers, kept in (([0, 1, 2], 0), ([1, 2], None), ([0, 2], None), ([2], None), ([], None)):
        pool = Pool([70, 0, 0], [2, 0, 0], [[4, 9, -1], [-1] * 3, [-1] * 3], [4, 9, 0, 1, 2, 3, 5, 6, 7, 8], 2, 10)
        d = Device(pool)
        pool.fork([-1, 0, 0])
        m.op_cache_fork(i32([-1, 0, 0]), d.seq, d.held, d.tables, d.shares)
        new = [int(s in writers) for s in range(3)]
        status, pairs = pool.own(new, 3)
        got = m.op_cache_own(d.seq, i32(new), d.held, d.free, d.head, d.tables, d.shares, 3)
        d.check(pool, status, pairs, got)
        assert len(pairs) == len(writers) - (kept is not None)
        if kept is not None:
            assert pool.tables[kept, 1] == 9


def test_fork_failures_change_nothing():
    m = lede()
    r = np.random.default_rng(4)
    base = _pool(r, 1400, 150, empty=0.5, spare=4000)
    source, lens = _forks(r, base)
    forks, parents = np.nonzero(source >= 0)[0], np.nonzero((source == -1) & (base.held > 0))[0]
    for at in (forks[0], forks[len(forks) // 2], forks[-1]):
        for what in ("source", "self", "chain", "low", "lens", "longer", "held", "parent"):
            say("fork failure", at, what)
            pool, src, ln = base.copy(), source.copy(), lens.copy()
            if what == "source":
                src[at] = 1400
            elif what == "self":
                src[at] = at
            elif what == "low":
                src[at] = -2
            elif what == "chain":
                src[at] = forks[1] if at != forks[1] else forks[0]
            elif what == "lens":
                ln[at] = -1
            elif what == "longer":
                ln[at] = pool.seq[src[at]] + 1
            elif what == "held":
                pool.held[at], pool.tables[at, 0] = 1, pool.free[-1]
            else:
                pool.seq[src[at]] = 64 * pool.held[src[at]] + 1
            d = Device(pool)
            want = pool.fork(src, ln)
            assert want[0] != 0
            assert m.op_cache_fork(i32(src), d.seq, d.held, d.tables, d.shares, lens=i32(ln)).tolist() == want
            d.check(pool)
    assert len(parents)


def test_own_failures_change_nothing():
    m = lede()
    r = np.random.default_rng(6)
    base = _pool(r, 1300, 190, extra=1, empty=0.6, spare=1500)
    source, _ = _forks(r, base, share=0.9)
    base.fork(source)
    new = r.integers(0, 100, 1300)
    full = base.copy()
    ok, all_pairs = full.own(new, 1300)
    need = ok[2] - base.head
    assert ok[0] == 0 and need > 300
    for change in ("new", "seq", "held", "head", "pages", "moves", "none"):
        say("own failure", change)
        pool, nw, moves = base.copy(), new.copy(), 1300
        if change == "new":
            nw[700] = -1
        elif change == "seq":
            pool.seq[1299] = -1
        elif change == "held":
            pool.held[3] = pool.tables.shape[1] + 1
        elif change == "head":
            pool.head = len(pool.free) + 1
        elif change == "pages":
            pool.free = pool.free[:pool.head + need - 1]
        elif change == "moves":
            moves = len(all_pairs) - 1
        else:
            moves = 0
        if change == "held":      # (the counterpart's holders would read past the row)
            held, pool.held[3] = pool.held[3], 0
            d = Device(pool)
            d.held[3] = int(held)
            want, pairs = [-1, 0, pool.head, 3], []
        else:
            d = Device(pool)
            want, pairs = pool.own(nw, moves)
        assert want[0] != 0
        got = m.op_cache_own(d.seq, i32(nw), d.held, d.free, d.head, d.tables, d.shares, moves)
        if change == "held":
            d.held[3] = 0
        d.check(pool, want, pairs, got)


@pytest.mark.parametrize("n,ctx,gone", [(1, 1, 1.0), (1, 64, 0.0), (5, 400, 0.5), (64, 4000, 0.1), (64, 20000, 0.5), (1023, 100, 0.5), (1025, 300, 1.0),
                                        (2100, 64, 0.3), (2100, 1500, 0.7), (2, 60000, 0.5), (2, 600000, 1.0)])
def test_free(n, ctx, gone):
    m = lede()
    for seed in range(2):
        say("free n=%d ctx=%d gone=%g seed=%d" % (n, ctx, gone, seed))
        r = np.random.default_rng(seed + 10 * n)
        pool = _pool(r, n, ctx, extra=2, empty=0.4)
        source, lens = _forks(r, pool)
        pool.fork(source, lens)
        pool.seq = np.where(r.random(n) < gone, 0, np.maximum(pool.seq - r.integers(0, 130, n), 0))
        d = Device(pool)
        for _ in range(2):
            want = pool.release()
            got = m.op_cache_free(d.seq, d.held, d.free, d.head, d.tables, d.shares, status=d.status)
            assert want[0] == 0 and got.tolist() == want
            d.check(pool)
        assert want[1] == 0


@pytest.mark.parametrize("n", [40, 1200])     # in one launch and in two
def test_free_failures_change_nothing(n):
    m = lede()
    r = np.random.default_rng(8)
    base = _pool(r, n, 300 if n > 100 else 2000, extra=1, empty=0.3)
    source, lens = _forks(r, base)
    base.fork(source, lens)
    base.seq[:] = base.seq // 3
    gone = base.copy().release()[1]
    for change in ("seq", "held", "head", "room", "low"):
        say("free failure", change)
        pool = base.copy()
        if change == "seq":
            pool.seq[n // 2] = -5
        elif change == "head":
            pool.head = len(pool.free) + 1
        elif change == "low":
            pool.head = -1
        elif change == "room":
            pool.head = gone - 1
        if change == "held":
            at = n - 3
            held, pool.held[at] = pool.tables.shape[1] + 1, 0
            d = Device(pool)
            d.held[at] = held
            want = [-1, 0, pool.head, at]
        else:
            d = Device(pool)
            want = pool.release()
        assert want[0] != 0
        assert m.op_cache_free(d.seq, d.held, d.free, d.head, d.tables, d.shares).tolist() == want
        if change == "held":
            d.held[at] = 0
        d.check(pool)


@pytest.mark.parametrize("n,ctx,spare", [(1, 1, 0), (1, 64, 5), (2, 500, 0), (9, 900, 300), (64, 3000, 1), (1025, 200, 4000), (2, 100, 262144 - 4), (7, 2000, 31)])
def test_compact(n, ctx, spare):
    m = lede()
    r = np.random.default_rng(n + ctx)
    say("compact n=%d ctx=%d spare=%d" % (n, ctx, spare))
    pool = _pool(r, n, ctx, extra=1, spare=max(spare, 1), empty=0.3)
    if n == 2 and spare > 100000:
        pool.n_pages = 262144
        pool.free = r.permutation(262144)
        pool.tables[pool.tables >= 0] = r.choice(262144, int((pool.tables >= 0).sum()), replace=False)
    source, lens = _forks(r, pool)
    pool.fork(source, lens)
    d = Device(pool)
    room = pool.n_pages // 2
    for again in range(2):
        want, pairs = pool.compact(room)
        got = m.op_cache_compact(d.held, d.free, d.head, d.tables, d.shares, room)
        assert want[0] == 0
        d.check(pool, want, pairs, got)
        d.head.copy_(got.status[2:3])
    assert not pairs


def test_compact_failures_change_nothing():
    m = lede()
    r = np.random.default_rng(12)
    base = _pool(r, 300, 400, spare=900)
    moves = len(base.copy().compact(10 ** 6)[1])
    for change in ("held", "low", "moves", "none", "list"):
        say("compact failure", change)
        pool, room = base.copy(), 10 ** 4
        if change == "moves":
            room = moves - 1
        elif change == "none":
            room = 0
        elif change == "list":
            pool.free = pool.free[:899]
            pool.head = 0
        if change in ("held", "low"):
            bad = pool.tables.shape[1] + 1 if change == "held" else -1
            pool.held[5] = 0
            d = Device(pool)
            d.held[5] = bad
            want, pairs = [-1, 0, pool.head, 5], []
        else:
            d = Device(pool)
            want, pairs = pool.compact(room)
        assert want[0] != 0
        got = m.op_cache_compact(d.held, d.free, d.head, d.tables, d.shares, room)
        if change in ("held", "low"):
            d.held[5] = 0
        d.check(pool, want, pairs, got)


def test_entries_outside_the_pool_are_left_alone():
    """Passed on by a fork, not counted, not freed, not moved."""
    m = lede()
    pool = Pool([130, 0, 65], [3, 0, 2], [[2, -1, 1 << 30], [-3] * 3, [5, -9, 0]], [0, 1, 3, 4, 2, 5], 0, 6)
    pool.tables[2, 1] = 6
    d = Device(pool)
    assert pool.fork([-1, 0, -1]) == [0, 3, -1]
    assert m.op_cache_fork(i32([-1, 0, -1]), d.seq, d.held, d.tables, d.shares).tolist() == [0, 3, -1]
    d.check(pool)
    status, pairs = pool.own([1, 1, 1], 3)
    d.check(pool, status, pairs, m.op_cache_own(d.seq, i32([1, 1, 1]), d.held, d.free, d.head, d.tables, d.shares, 3))
    status, pairs = pool.compact(3)
    got = m.op_cache_compact(d.held, d.free, d.head, d.tables, d.shares, 3)
    d.check(pool, status, pairs, got)
    d.head.copy_(got.status[2:3])
    pool.seq[:] = 0
    d.seq.zero_()
    assert m.op_cache_free(d.seq, d.held, d.free, d.head, d.tables, d.shares).tolist() == pool.release()
    d.check(pool)


def test_own_of_pages_that_are_listed_as_free():
    """A list that is wrong gives wrong pages, but no more of them than there are, and no pair behind the last."""
    m = lede()
    n = 128
    tables = [[2 * (s // 2), 2 * (s // 2) + 1] for s in range(n)]          # two sequences share two pages
    for order in (list(range(n)), list(range(n - 1, -1, -1))):
        pool = Pool([70] * n, [2] * n, tables, order, n // 2, n)
        d = Device(pool)
        d.shares.fill_(1)
        pairs = torch.full((2 * n + 64,), 12345, dtype=torch.int32, device="cuda")
        out = m.CacheMoves(pairs[:n].view(n // 2, 2), torch.empty(4, dtype=torch.int32, device="cuda"))
        m.op_cache_own(d.seq, i32([10] * n), d.held, d.free, d.head, d.tables, d.shares, n // 2, out=out)
        assert out.status.tolist() == [0, n // 2, n, -1]
        assert bool((pairs[n:] == 12345).all()) and bool((out.pairs < n).all())
        for name, g in d.guards.items():
            assert bool((g == 12345).all()), name


@pytest.mark.parametrize("kv,hd,n_pages", [(1, 64, 5), (4, 64, 300), (8, 128, 40), (3, 128, 33), (40, 128, 9), (1024, 64, 3)])
def test_copy(kv, hd, n_pages):
    m = lede()
    say("copy kv=%d hd=%d pages=%d" % (kv, hd, n_pages))
    r = np.random.default_rng(kv)
    nbytes = m.load().lede_op_cache_bytes(n_pages, kv, hd)
    flat = torch.randint(0, 256, (nbytes + 64,), dtype=torch.uint8, device="cuda")
    cache = m.Cache(n_pages, kv, hd, region=flat[:nbytes])
    order = r.permutation(n_pages)
    k = n_pages // 2
    pairs = [(int(a), int(b)) for a, b in zip(order[:k], order[k:])]
    pairs[0:0] = [(-1, int(order[0])), (int(order[0]), n_pages)]        # skipped
    for count in (0, 1, len(pairs), len(pairs) + 5, -3):
        want, size = flat.clone(), kv * PAGE * hd
        for a, b in pairs[:max(count, 0)]:
            if 0 <= a < n_pages and 0 <= b < n_pages:
                for at, w in ((0, size), (n_pages * size, size), (2 * n_pages * size, 8 * kv)):
                    want[at + b * w:at + (b + 1) * w] = want[at + a * w:at + (a + 1) * w].clone()
        m.op_cache_copy(cache, i32(pairs).view(-1, 2), i32([count]))
        assert torch.equal(flat, want), count


def test_copy_past_4_gib():
    m = lede()
    kv, hd = 8, 128
    n_pages = (1 << 32) // (kv * PAGE * hd) + 40
    cache = m.Cache(n_pages, kv, hd)
    say("copy in a cache of %.1f GiB" % (cache.region.numel() / 2 ** 30))
    size = kv * PAGE * hd
    a, b = n_pages - 2, n_pages - 17
    for at, w in ((0, size), (n_pages * size, size), (2 * n_pages * size, 8 * kv)):
        cache.region[at + a * w:at + (a + 1) * w] = torch.randint(1, 256, (w,), dtype=torch.uint8, device="cuda")
    m.op_cache_copy(cache, i32([[a, b]]), i32([1]))
    for at, w in ((0, size), (n_pages * size, size), (2 * n_pages * size, 8 * kv)):
        assert torch.equal(cache.region[at + a * w:at + (a + 1) * w], cache.region[at + b * w:at + (b + 1) * w])
        assert not cache.region[at + b * w:at + (b + 1) * w].eq(0).any()


# ---- together ---------------------------------------------------------------------------------


class Server:
    """Requests over one cache: every pass plans, appends and attends; forks, rollbacks, ends and compactions between."""

    def __init__(self, seed, seqs=6, kv=2, hd=64, n_pages=40, width=6):
        m = lede()
        self.r, self.seqs, self.kv, self.hd, self.n_pages = np.random.default_rng(seed), seqs, kv, hd, n_pages
        self.cache = m.Cache(n_pages, kv, hd)
        self.seq, self.held = i32(np.zeros(seqs)), i32(np.zeros(seqs))
        self.tables, self.shares = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda"), i32(np.zeros(n_pages))
        self.free, self.status = i32(self.r.permutation(n_pages)), i32([0, 0, 0, -1])
        self.head = self.status[2:3]
        self.moves = m.CacheMoves(torch.empty(n_pages, 2, dtype=torch.int32, device="cuda"), self.status)

    def append(self, new, k, v, q, plan):
        m = lede()
        m.op_cache_own(self.seq, new, self.held, self.free, self.head, self.tables, self.shares, self.n_pages, out=self.moves)
        m.op_cache_copy(self.cache, self.moves.pairs, self.moves.status[1:2])
        m.op_cache_plan(self.seq, new, self.held, self.free, self.head, self.tables, plan.slots.numel(), out=plan)
        m.op_cache_append(self.cache, k, v, plan.slots)
        return m.op_cache_attention(self.cache, q, self.tables, plan.kv_lens, plan.row_start, 64, 64 * self.tables.shape[1])

    def plan(self, rows):
        return lede().CachePlan(self.seq, self.held, torch.zeros(self.seqs + 1, dtype=torch.int32, device="cuda"),
                                torch.empty(rows, dtype=torch.int64, device="cuda"), self.status)


def test_server_run():
    """Each request's tokens stay its own through forks, rollbacks, ends and compactions: what its pages hold is what a
    cache of its own would."""
    m = lede()
    sv = Server(3)
    r = np.random.default_rng(7)
    mine = [np.zeros((0, 2, sv.kv, sv.hd)) for _ in range(sv.seqs)]
    small = lambda n: np.ldexp(r.integers(-7, 8, (n, 2, sv.kv, sv.hd)), -3).astype(np.float64)  # noqa: E731  (exact in every block)
    for step in range(40):
        say("server step", step)
        what = step % 5
        if what == 1:        # forks of whole requests and of prefixes, into those that are empty
            source, lens = np.full(sv.seqs, -1), np.zeros(sv.seqs, int)
            parents = [s for s in range(sv.seqs) if len(mine[s])]
            for s in range(sv.seqs):
                if len(mine[s]) == 0 and parents and int(sv.held[s]) == 0:
                    source[s] = r.choice(parents)
                    lens[s] = len(mine[source[s]]) if r.random() < 0.5 else r.integers(0, len(mine[source[s]]) + 1)
                    mine[s] = mine[source[s]][:lens[s]].copy()
            assert m.op_cache_fork(i32(source), sv.seq, sv.held, sv.tables, sv.shares, lens=i32(lens))[0].item() == 0
        elif what == 3:      # rollbacks and ends; spare pages given back every other time
            for s in range(sv.seqs):
                n = 0 if r.random() < 0.4 else max(0, len(mine[s]) - int(r.integers(0, 70)))
                mine[s] = mine[s][:n]
            sv.seq.copy_(i32([len(x) for x in mine]))
            if step % 2 or sum(len(x) == 0 for x in mine):
                m.op_cache_free(sv.seq, sv.held, sv.free, sv.head, sv.tables, sv.shares, status=sv.status)
                assert sv.status[0].item() == 0
        elif what == 4:
            m.op_cache_compact(sv.held, sv.free, sv.head, sv.tables, sv.shares, sv.n_pages, out=sv.moves)
            m.op_cache_copy(sv.cache, sv.moves.pairs, sv.moves.status[1:2])
            assert sv.status[0].item() == 0
        new = np.minimum(r.integers(0, 40, sv.seqs), 300 - np.array([len(x) for x in mine]))
        rows = int(new.sum())
        x = small(rows + 1)
        at = 0
        for s in range(sv.seqs):
            mine[s] = np.concatenate([mine[s], x[at:at + new[s]]])
            at += new[s]
        d = torch.from_numpy(x).to("cuda").to(torch.bfloat16)
        q = torch.zeros(rows + 1, sv.kv, sv.hd, dtype=torch.bfloat16, device="cuda")
        plan = sv.plan(rows + 1)
        out = sv.append(i32(new), d[:, 0], d[:, 1], q, plan)
        assert sv.status[0].item() == 0
        tables, held, seq = sv.tables.cpu().numpy(), sv.held.cpu().numpy(), sv.seq.cpu().numpy()
        assert seq.tolist() == [len(v) for v in mine]
        state = Pool(seq, held, tables, sv.free.cpu().numpy(), int(sv.head), sv.n_pages)
        assert np.array_equal(sv.shares.cpu().numpy(), state.shares())
        # every page is either held or free, once
        free = state.free[state.head:]
        assert sorted(free.tolist() + np.nonzero(state.holders())[0].tolist()) == list(range(sv.n_pages))
        start = plan.row_start.cpu().numpy()
        for s in range(sv.seqs):
            p = np.arange(len(mine[s]))
            slots = torch.from_numpy(tables[s, p // PAGE].astype(np.int64) * PAGE + p % PAGE).to("cuda")
            k, v = m.op_cache_read(sv.cache, slots, torch.float32)
            assert np.array_equal(k.double().cpu().numpy(), mine[s][:, 0]) and np.array_equal(v.double().cpu().numpy(), mine[s][:, 1])
            for i in range(new[s]):     # queries of zeros: the mean of the values seen
                seen = len(mine[s]) - new[s] + i + 1
                got = out[start[s] + i].double().cpu().numpy()
                want = mine[s][:seen, 1].mean(0)
                assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -11).all()


def test_server_in_a_graph():
    """A captured pass of own, copy, plan, append and attention, replayed between eager forks, frees and compactions."""
    m = lede()
    eager, sv = Server(5), Server(5)
    rows = 12
    new = i32([2, 0, 3, 1, 4, 2])
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.zeros(rows, 2, 64, dtype=torch.bfloat16, device="cuda")
    v, q = torch.zeros_like(k), torch.zeros_like(k)
    plans = eager.plan(rows), sv.plan(rows)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        res = sv.append(new, k, v, q, plans[1])
    for step in range(24):
        for t in (k, v, q):
            t.normal_(generator=g)
        if step % 6 == 3:
            for x in (eager, sv):
                x.seq[5:].zero_()
                m.op_cache_free(x.seq, x.held, x.free, x.head, x.tables, x.shares, status=x.status)
                assert m.op_cache_fork(i32([-1] * 5 + [2]), x.seq, x.held, x.tables, x.shares)[0].item() == 0
        if step % 6 == 5:
            for x in (eager, sv):
                x.seq.copy_((x.seq - 20).clamp(min=0))
                m.op_cache_free(x.seq, x.held, x.free, x.head, x.tables, x.shares, status=x.status)
                m.op_cache_compact(x.held, x.free, x.head, x.tables, x.shares, x.n_pages, out=x.moves)
                m.op_cache_copy(x.cache, x.moves.pairs, x.moves.status[1:2])
        want = eager.append(new, k, v, q, plans[0])
        graph.replay()
        torch.cuda.synchronize()
        assert int(sv.status[0]) == 0
        for a, b in ((eager.seq, sv.seq), (eager.held, sv.held), (eager.shares, sv.shares), (eager.free, sv.free), (eager.status, sv.status),
                     (eager.moves.pairs, sv.moves.pairs), (plans[0].slots, plans[1].slots), (want, res)):
            assert torch.equal(a, b), step
        for s in range(6):
            h = int(sv.held[s])
            assert torch.equal(eager.tables[s, :h], sv.tables[s, :h])


def test_calls_on_another_stream():
    m = lede()
    r = np.random.default_rng(31)
    pool = _pool(r, 300, 900, empty=0.5, spare=800)
    source, lens = _forks(r, pool)
    d = Device(pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        src, ln, new = i32(source), i32(lens), i32(np.ones(300))
        m.op_cache_fork(src, d.seq, d.held, d.tables, d.shares, lens=ln)
        mv = m.op_cache_own(d.seq, new, d.held, d.free, d.head, d.tables, d.shares, 300)
    torch.cuda.current_stream().wait_stream(side)
    pool.fork(source, lens)
    status, pairs = pool.own(np.ones(300, int), 300)
    d.check(pool, status, pairs, mv)
    assert ref.OK == status[0] and pages(65) == 2
