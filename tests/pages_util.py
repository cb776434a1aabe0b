"""A plain model of the page calls: one sequence, entry and page after another, on the host."""
import numpy as np


def n_pages_of(length, page):
    return -(-max(int(length), 0) // page)


class Model:
    """lens, refs and table as lists; each call does what its definition says, in order."""

    def __init__(self, B, max_pages, n_pages, page):
        self.B, self.max_pages, self.n_pages, self.page = B, max_pages, n_pages, page
        self.lens = [0] * B
        self.refs = [0] * n_pages
        self.table = [[-1] * max_pages for _ in range(B)]

    def fork(self, parent):
        lens, table = list(self.lens), [list(r) for r in self.table]
        for b, src in enumerate(parent):
            ok = 0 <= src < self.B
            self.lens[b] = lens[src] if ok else 0
            self.table[b] = list(table[src]) if ok else [-1] * self.max_pages
        self.count()

    def count(self):
        self.refs = [0] * self.n_pages
        for row in self.table:
            for p in row:
                if p >= 0:
                    self.refs[p] += 1

    def reserve(self, n_new):
        """(starts, granted, moves, info)"""
        starts, n_new = list(self.lens), [max(int(n), 0) for n in n_new]
        refs, table = list(self.refs), [list(r) for r in self.table]
        free = [p for p in range(self.n_pages) if refs[p] <= 0]
        need, over, moves, taken = 0, 0, [], []
        for b, n in enumerate(n_new):
            if n == 0:
                continue
            had, has = n_pages_of(starts[b], self.page), n_pages_of(starts[b] + n, self.page)
            if has > self.max_pages:
                over += 1
            slots = list(range(had, has))
            if starts[b] % self.page and refs[table[b][had - 1]] > 1:
                slots.insert(0, had - 1)
            for s in slots:
                need += 1
                if s >= self.max_pages or len(taken) == len(free):
                    if s == had - 1:
                        refs[table[b][s]] -= 1
                    continue
                p = free[len(taken)]
                taken.append(p)
                if s == had - 1:
                    moves.append((table[b][s], p))
                    refs[table[b][s]] -= 1
                table[b][s] = p
                refs[p] = 1
        if over or need > len(free):
            return starts, [0] * self.B, [], [0, 0, max(need - len(free), 0), over]
        self.refs, self.table = refs, table
        self.lens = [a + n for a, n in zip(starts, n_new)]
        return starts, n_new, moves, [len(moves), need, 0, 0]

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        high = [p for p in range(live, self.n_pages) if self.refs[p] > 0]
        to = dict(zip(high, holes))
        for src, dst in to.items():
            self.refs[dst], self.refs[src] = self.refs[src], 0
        self.table = [[to.get(p, p) for p in r] for r in self.table]
        return list(to.items()), [len(to), live, 0, 0]


def filled(rng, B, max_pages, n_pages, page, share=0.5, order=None):
    """A model in which sequences of random lengths were grown, some of them forks of others."""
    m = Model(B, max_pages, n_pages, page)
    order = rng.permutation(n_pages) if order is None else order
    free = [int(p) for p in order]
    for b in range(B):
        if b and rng.random() < share:
            src = int(rng.integers(b))
            m.lens[b], m.table[b] = m.lens[src], list(m.table[src])
            if rng.random() < 0.4 and m.lens[b]:  # a fork that went on alone: its last page is its own
                if not free:
                    continue
                m.table[b][n_pages_of(m.lens[b], page) - 1] = free.pop()
            continue
        length = int(rng.integers(0, max_pages * page + 1))
        length = min(length, len(free) * page)
        m.lens[b] = length
        for j in range(n_pages_of(length, page)):
            m.table[b][j] = free.pop()
    m.count()
    return m


def to_device(m, torch):
    from paper_2607_07740_amd import api
    dev = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    return api.PageTable(dev(m.lens), dev(m.refs), dev(m.table).view(m.B, m.max_pages), m.page)


def same(pages, m):
    assert pages.lens.tolist() == m.lens
    assert pages.refs.tolist() == m.refs
    assert pages.table.tolist() == m.table
