"""The pages of paged caches on the host, by their definitions, page by page (used by the tests of the page calls)."""
import random

import torch

POOL_FULL, BAD_SEQ, BAD_PAGE = 128, 256, 32


class Pool:
    """refs, table (rows of any length are padded with -1), held, len."""

    def __init__(self, n_pages, page, n_seqs, table_ld):
        self.n_pages, self.page, self.n_seqs, self.table_ld = n_pages, page, n_seqs, table_ld
        self.refs, self.held, self.len = [0] * n_pages, [0] * n_seqs, [0] * n_seqs
        self.table = [[-1] * table_ld for _ in range(n_seqs)]
        self.status = 0

    @classmethod
    def random(cls, seed, n_pages, page, n_seqs, table_ld, fill=0.6, external=0):
        """Sequences of any length on pages in any order; some hold pages beyond their tokens."""
        p, r = cls(n_pages, page, n_seqs, table_ld), random.Random(seed)
        order = list(range(n_pages))
        r.shuffle(order)
        budget = int(n_pages * fill)
        for b in r.sample(range(n_seqs), n_seqs):
            h = min(r.randint(0, table_ld), budget)
            budget -= h
            for i in range(h):
                p.table[b][i] = order.pop()
                p.refs[p.table[b][i]] += 1
            p.held[b] = h
            p.len[b] = r.randint(0, h * page) if r.random() < 0.4 else max(0, h * page - r.randint(0, page))
        for _ in range(external):
            p.refs[r.randrange(n_pages)] += 1
        return p

    def pages_of(self, tokens):
        return -(-tokens // self.page)

    def fork(self, parent, keep=None):
        rows, lens, helds = [list(x) for x in self.table], list(self.len), list(self.held)
        for b, par in enumerate(parent):
            if par >= self.n_seqs:
                self.status |= BAD_SEQ
                continue
            n = 0 if par < 0 else lens[par] if keep is None else min(lens[par], max(0, keep[b]))
            if par == b and n == lens[b] and keep is None:
                continue
            h = 0 if par < 0 else min(self.pages_of(n), helds[par])
            for i in range(helds[b]):
                self.refs[rows[b][i]] -= 1
                self.table[b][i] = -1
            for i in range(h):
                self.table[b][i] = rows[par][i]
                self.refs[rows[par][i]] += 1
            self.len[b], self.held[b] = n, h

    def extend(self, rows):
        """The copies; None: it cannot be served."""
        P = self.page
        writes = {}                                     # page: sequences that write it
        for b, r in enumerate(rows):
            if r > 0:
                for i in range(self.len[b] // P, min(self.held[b], self.pages_of(self.len[b] + r))):
                    writes.setdefault(self.table[b][i], []).append(b)
        new, copies, free = [], [], [p for p in range(self.n_pages) if self.refs[p] == 0]
        for b, r in enumerate(rows):
            if r <= 0:
                continue
            need = self.pages_of(self.len[b] + r)
            if need > self.table_ld:
                self.status |= POOL_FULL
                return None
            for i in range(self.len[b] // P, min(self.held[b], need)):
                page = self.table[b][i]
                who = writes[page]
                if self.refs[page] > 1 and not (len(who) == self.refs[page] and who[-1] == b):
                    new.append((b, i, page))
            new += [(b, i, None) for i in range(self.held[b], need)]
        if len(new) > len(free):
            self.status |= POOL_FULL
            return None
        for (b, i, was), page in zip(new, free):
            if was is not None:
                self.refs[was] -= 1
                if i == self.len[b] // P and self.len[b] % P:
                    copies.append((was, page, self.len[b] % P))
            else:
                self.held[b] = i + 1
            self.refs[page] = 1
            self.table[b][i] = page
        return copies

    def compact(self):
        used = [p for p in range(self.n_pages) if self.refs[p] > 0]
        n = len(used)
        moves = dict(zip([p for p in used if p >= n], [p for p in range(n) if self.refs[p] == 0]))
        for a, b in moves.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for b in range(self.n_seqs):
            for i in range(self.held[b]):
                self.table[b][i] = moves.get(self.table[b][i], self.table[b][i])
        return [(a, b, self.page) for a, b in moves.items()]

    def used(self):
        return sum(r > 0 for r in self.refs)


class DevicePool:
    def __init__(self, pool, device="cuda:0"):
        import paper_2502_09888_amd as P
        self.P, self.c = P, pool

        def ints(x):
            return torch.tensor(x, dtype=torch.int32, device=device)
        self.ints = ints
        self.refs, self.table, self.held, self.len = ints(pool.refs), ints(pool.table), ints(pool.held), ints(pool.len)
        self.pool = P.page_pool(self.refs, self.table, self.held, self.len, pool.page)
        self.copies = torch.full((max(pool.n_seqs, pool.n_pages // 2, 1), 3), -9, dtype=torch.int32, device=device)
        self.counts, self.status = ints([-9, -9]), ints([0])
        self.ws = torch.full((P.climber_pages_workspace_bytes(self.pool),), 0xFF, dtype=torch.uint8, device=device)

    def fork(self, parent, keep=None, stream=None):
        self.P.climber_pages_fork(self.pool, self.ints(parent), None if keep is None else self.ints(keep), self.status, self.ws, stream)

    def extend(self, rows, stream=None):
        self.copies.fill_(-9)
        self.P.climber_pages_extend(self.pool, self.ints(rows), self.copies, self.counts, self.status, self.ws, stream)

    def compact(self, stream=None):
        self.copies.fill_(-9)
        self.P.climber_pages_compact(self.pool, self.copies, self.counts, self.status, self.ws, stream)

    def check(self, copies=None):
        """Against the pool on the host; `copies`: those of the last call that makes any."""
        torch.cuda.synchronize()
        c = self.c
        assert self.refs.tolist() == c.refs and self.held.tolist() == c.held and self.len.tolist() == c.len
        assert self.table.tolist() == c.table
        assert self.status.item() == c.status
        if copies is not None:
            assert self.counts.tolist() == [len(copies), c.used()]
            got = self.copies.tolist()
            assert [tuple(x) for x in got[:len(copies)]] == copies and all(x == [-9] * 3 for x in got[len(copies):])
