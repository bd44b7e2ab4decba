"""Plain counterparts of the calls that share, own, free and compact the pages of a batch's cache: one sequence after the
other, with the holders of every page counted anew from the tables."""
import numpy as np

PAGE = 64
OK, E_ARG, E_STATE, E_KV_FULL = 0, -1, -2, -3


def pages(tokens):
    return -(-int(tokens) // PAGE)


class Pool:
    """Lengths, tables and the free list; free pages are free_pages[head:]."""

    def __init__(self, seq_lens, held, tables, free_pages, head, n_pages):
        self.seq, self.held = np.array(seq_lens, np.int64), np.array(held, np.int64)
        self.tables, self.free, self.head, self.n_pages = np.array(tables, np.int64), np.array(free_pages, np.int64), int(head), n_pages

    def copy(self):
        return Pool(self.seq, self.held, self.tables, self.free, self.head, self.n_pages)

    def entries(self):
        for s in range(len(self.seq)):
            for i in range(self.held[s]):
                if 0 <= self.tables[s, i] < self.n_pages:
                    yield s, i, int(self.tables[s, i])

    def holders(self):
        n = np.zeros(self.n_pages, np.int64)
        for _, _, p in self.entries():
            n[p] += 1
        return n

    def shares(self):
        return np.maximum(self.holders() - 1, 0)

    def fits(self, s):
        return self.seq[s] >= 0 and 0 <= self.held[s] <= self.tables.shape[1] and pages(self.seq[s]) <= self.held[s]

    def fork(self, source, lens=None):
        n = len(self.seq)
        for s in range(n):
            r = source[s]
            if r == -1:
                continue
            if not 0 <= r < n or r == s or source[r] != -1 or not self.fits(r) or (lens is not None and not 0 <= lens[s] <= self.seq[r]):
                return [E_ARG, 0, s]
            if self.held[s] != 0:
                return [E_STATE, 0, s]
        shared = 0
        for s in range(n):
            r = source[s]
            if r >= 0:
                self.seq[s] = self.seq[r] if lens is None else lens[s]
                self.held[s] = pages(self.seq[s])
                self.tables[s, :self.held[s]] = self.tables[r, :self.held[s]]
                shared += int(self.held[s])
        return [OK, shared, -1]

    def own(self, new, max_moves):
        n = len(self.seq)
        for s in range(n):
            if not 0 <= self.head <= len(self.free) or new[s] < 0 or not self.fits(s):
                return [E_ARG, 0, self.head, s], []
        holders, writes = self.holders(), []
        for s in range(n):
            if new[s]:
                for i in range(int(self.seq[s]) // PAGE, min(int(self.held[s]), pages(self.seq[s] + new[s]))):
                    if 0 <= self.tables[s, i] < self.n_pages:
                        writes.append((s, i, int(self.tables[s, i])))
        by_page = {}
        for s, i, p in writes:
            by_page.setdefault(p, []).append((s, i))
        head, pairs, new_entries = self.head, [], []
        for s, i, p in writes:
            if len(by_page[p]) == holders[p] and by_page[p][0] == (s, i):
                continue
            if head >= len(self.free):
                return [E_KV_FULL, 0, self.head, s], []
            if i * PAGE < self.seq[s]:
                pairs.append((p, int(self.free[head])))
                if len(pairs) > max_moves:
                    # a sequence fails as a whole: it takes all of its pages first
                    takes = sum(1 for t, j, q in writes if t == s and j > i and not (len(by_page[q]) == holders[q] and by_page[q][0] == (t, j)))
                    return [E_KV_FULL if head + 1 + takes > len(self.free) else E_ARG, 0, self.head, s], []
            new_entries.append((s, i, int(self.free[head])))
            head += 1
        for s, i, p in new_entries:
            self.tables[s, i] = p
        self.head = head
        return [OK, len(pairs), head, -1], pairs

    def release(self):
        n = len(self.seq)
        for s in range(n):
            if self.seq[s] < 0 or not 0 <= self.held[s] <= self.tables.shape[1] or not 0 <= self.head <= len(self.free):
                return [E_ARG, 0, self.head, s]
        before = self.holders()
        held = np.minimum(self.held, [pages(x) for x in self.seq])
        old, self.held = self.held, held
        gone = np.nonzero((before > 0) & (self.holders() == 0))[0]
        if len(gone) > self.head:
            self.held = old
            return [E_ARG, 0, self.head, -1]
        self.head -= len(gone)
        self.free[self.head:self.head + len(gone)] = gone
        return [OK, len(gone), self.head, -1]

    def compact(self, max_moves):
        for s in range(len(self.seq)):
            if not 0 <= self.held[s] <= self.tables.shape[1]:
                return [E_ARG, 0, self.head, s], []
        live = sorted({p for _, _, p in self.entries()})
        n = len(live)
        holes = sorted(set(range(n)) - set(live))
        pairs = list(zip([p for p in live if p >= n], holes))
        if len(pairs) > max_moves or len(self.free) < self.n_pages - n:
            return [E_ARG, 0, self.head, -1], []
        to = dict(pairs)
        for s, i, p in list(self.entries()):
            self.tables[s, i] = to.get(p, p)
        self.head = len(self.free) - (self.n_pages - n)
        self.free[self.head:] = np.arange(n, self.n_pages)
        return [OK, len(pairs), self.head, n], pairs
