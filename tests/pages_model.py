"""The paged cache's rules in plain Python lists (test infrastructure): what append, fork, free,
compact and commit do to tables, lengths, reference counts and contents."""
from __future__ import annotations

import numpy as np


class PoolModel:
    """contents[p][s]: whatever the slot holds (here: a number per token)."""

    def __init__(self, n_pages, page, n_seqs, table_ld, fill=-1.0):
        self.page, self.table_ld = page, table_ld
        self.table = [[] for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.refs = [0] * n_pages
        self.slots = np.full((n_pages, page), fill)

    def _free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def _need(self, b, rows):
        end = self.len[b] + rows
        if end > self.table_ld * self.page:
            return -1
        return -(-end // self.page) - (-(-self.len[b] // self.page))

    def _take(self, needs):
        """missing[i], and the pages that i gets."""
        free, total, missing, given = self._free_pages(), 0, [], []
        for n in needs:
            if n < 0:
                missing.append(-1)
                given.append([])
                continue
            total += n
            lack = min(n, max(0, total - len(free)))
            missing.append(lack)
            given.append(free[total - n:total] if lack == 0 else [])
        return missing, given

    def append(self, items):
        """items: (sequence, values of its new tokens)."""
        missing, given = self._take([self._need(b, len(v)) for b, v in items])
        for (b, values), lack, pages in zip(items, missing, given):
            if lack:
                continue
            for p in pages:
                self.refs[p] = 1
            self.table[b] += pages
            for x in values:
                t = self.len[b]
                self.slots[self.table[b][t // self.page], t % self.page] = x
                self.len[b] += 1
        return missing

    def free(self, seqs):
        for b in seqs:
            for p in self.table[b]:
                self.refs[p] -= 1
            self.table[b], self.len[b] = [], 0

    def fork(self, src, dst):
        self.free(dst)
        missing, given = self._take([1 if self.len[s] % self.page else 0 for s in src])
        for s, d, lack, pages in zip(src, dst, missing, given):
            if lack:
                continue
            full, rest = divmod(self.len[s], self.page)
            self.table[d] = self.table[s][:full] + pages
            self.len[d] = self.len[s]
            for p in self.table[s][:full]:
                self.refs[p] += 1
            for p in pages:
                self.refs[p] = 1
                self.slots[p, :rest] = self.slots[self.table[s][full], :rest]
        return missing

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r]
        n = len(live)
        to = dict(zip([p for p in live if p >= n], [p for p in range(n) if self.refs[p] == 0]))
        for a, b in to.items():
            self.slots[b] = self.slots[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return n

    def tokens(self, b):
        return [self.slots[self.table[b][t // self.page], t % self.page] for t in range(self.len[b])]


def walk(tokens, parents, chosen, n):
    """The confirmed path of one tree."""
    path = []
    cur = 0 if n else None
    while cur is not None:
        path.append(cur)
        cur = next((j for j in range(cur + 1, n) if parents[j] == cur and tokens[j] == chosen[cur]), None)
    return path
