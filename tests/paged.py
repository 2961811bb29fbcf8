"""A cache in pages for the tests: tables in no order, and plain models of the pages' bookkeeping, one entry after the other."""
import torch

DEV = "cuda:0"
PAGES = [16, 32, 64, 128, 256]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def table_of(rows, page, seed=0, spare=3, extra=1):
    """Page table for sequences of so many rows (and `extra` columns more), the number of pages, slots of every row of every sequence.  No page twice."""
    need = [-(-r // page) for r in rows]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = [[order.pop() for _ in range(n)] + [-1] * (max(need) + extra - n) for n in need]
    return table, n_pages, [slots_of(t, r, page) for t, r in zip(table, rows)]


def slots_of(entries, rows, page):
    return torch.tensor([entries[r // page] * page + r % page for r in range(rows)], dtype=torch.int64)


def pages_of(n, page):
    return -(-n // page)


class Model:
    """refs, free pages (the last is the next) and page tables on the host."""

    def __init__(self, n_pages, page):
        self.n, self.page = n_pages, page
        self.refs, self.free = [0] * n_pages, list(range(n_pages - 1, -1, -1))

    def fork(self, table, lens, parents):
        out, lens_out = [], []
        for p in parents:
            if not 0 <= p < len(table):
                out.append([-1] * len(table[0]))
                lens_out.append(0)
                continue
            n = pages_of(lens[p], self.page)
            out.append(table[p][:n] + [-1] * (len(table[p]) - n))
            lens_out.append(lens[p])
            for x in out[-1][:n]:
                self.refs[x] += 1
        return out, lens_out

    def reserve(self, table, first, to):
        """-> (ends, pairs of copied pages); changes the table."""
        room = len(table[0]) * self.page
        asked = [(s, i) for s, (a, b) in enumerate(zip(first, to)) if 0 <= a < b <= room for i in range(a // self.page, pages_of(b, self.page))]
        entries = [table[s][i] for s, i in asked]
        # of the holders of a page that all ask for it the last keeps it
        keeps = {p: asked[len(entries) - 1 - entries[::-1].index(p)] for p in set(entries) if p >= 0 and entries.count(p) == self.refs[p]}
        need = {s: [i for r, i in asked if r == s and (table[s][i] < 0 or keeps.get(table[s][i]) != (s, i))] for s, _ in asked}
        ends, pairs, wanted, had = [], [], 0, len(self.free)
        for s, (a, b) in enumerate(zip(first, to)):
            if s not in need:
                ends.append(a)
                continue
            wanted += len(need[s])
            if wanted <= had:
                for i in need[s]:
                    new = self.free.pop()
                    if table[s][i] >= 0:
                        self.refs[table[s][i]] -= 1
                        pairs.append((table[s][i], new))
                    self.refs[new] = 1
                    table[s][i] = new
                ends.append(b)
            else:
                alone = all(table[s][i] >= 0 and self.refs[table[s][i]] == 1 for r, i in asked if r == s)
                ends.append(b if not need[s] and alone else a)
        return ends, pairs

    def release(self, table, keep):
        freed = []
        for row, k in zip(table, keep):
            for i in range(pages_of(max(k, 0), self.page), len(row)):
                if row[i] >= 0:
                    self.refs[row[i]] -= 1
                    freed.append(row[i])
                    row[i] = -1
        last = {p: at for at, p in enumerate(freed)}
        self.free += [p for at, p in enumerate(freed) if self.refs[p] == 0 and last[p] == at][::-1]
