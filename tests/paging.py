"""Plain Python models of the paged cache and its page bookkeeping (test infrastructure)."""
from __future__ import annotations

import torch


def pages_of(tokens, P):
    return -(-tokens // P)


def to_pages(cache, lens, P, n, seed, spare=3, width=None, fill=float("nan")):
    """A contiguous cache [B][Lcap*n][Hkv][Dh] cut into pages that lie in random order in a pool.  Every row
    that no sequence holds (free pages, rows behind a sequence's tokens) is `fill`.  Returns (pool, page_table)."""
    B, _, Hkv, Dh = cache.shape
    held = [pages_of(int(x), P) for x in lens]
    pages = sum(held) + spare
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    pool = torch.full((pages, P * n, Hkv, Dh), fill, dtype=cache.dtype)
    table = torch.full((B, width or max(1, max(held))), -1, dtype=torch.int32)
    for b, T in enumerate(int(x) for x in lens):
        for i in range(held[b]):
            table[b, i] = pg = perm.pop()
            rows = cache[b, i * P * n:min((i + 1) * P, T) * n]
            pool[pg, :rows.shape[0]] = rows
    return pool, table


def rows_of(pool, table_row, tokens, n):
    """The first tokens * n rows of a sequence, from its pages."""
    P = pool.shape[1] // n
    ids = table_row[:pages_of(tokens, P)].long()
    return pool[ids].flatten(0, 1)[:tokens * n]


class Book:
    """Who holds which page, step by step in the order that the header gives."""
    INDEX, PAGES = 1, 4

    def __init__(self, B, width, pages, P):
        self.refs, self.table, self.lens = [0] * pages, [[-1] * width for _ in range(B)], [0] * B
        self.B, self.width, self.pages, self.P, self.status = B, width, pages, P, 0

    def _take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def grow(self, add):
        left, asked = self.refs.count(0), 0
        for b, x in enumerate(add):
            if x < 0 or self.lens[b] + x > self.width * self.P:
                self.status |= self.INDEX
                continue
            have, want = pages_of(self.lens[b], self.P), pages_of(self.lens[b] + x, self.P)
            asked += want - have
            if want > have and asked > left:
                self.status |= self.PAGES
                continue
            # those served come first in the order of free ids, so taking the lowest one is the same
            for i in range(have, want):
                self.table[b][i] = self._take()
            self.lens[b] += x

    def fork(self, src, dst, tokens=None):
        copies, seen, lens0 = [], set(), list(self.lens)
        for i, (a, b) in enumerate(zip(src, dst)):
            copies.append((-1, -1))
            first = b not in seen
            seen.add(b)
            ok = 0 <= a < self.B and 0 <= b < self.B and a != b and first and lens0[b] == 0
            t = 0
            if ok:
                t = lens0[a] if tokens is None else tokens[i]
                ok = 0 <= t <= lens0[a]
            if not ok:
                self.status |= self.INDEX
                continue
            full = t // self.P
            if t % self.P:
                if 0 not in self.refs:
                    self.status |= self.PAGES
                    continue
                self.table[b][full] = p = self._take()
                copies[-1] = (self.table[a][full], p)
            for j in range(full):
                self.table[b][j] = self.table[a][j]
                self.refs[self.table[a][j]] += 1
            self.lens[b] = t
        return copies

    def free(self, seqs):
        for b in seqs:
            if not 0 <= b < self.B:
                self.status |= self.INDEX
                continue
            for i in range(pages_of(self.lens[b], self.P)):
                self.refs[self.table[b][i]] -= 1
                self.table[b][i] = -1
            self.lens[b] = 0

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        K = len(live)
        moves = list(zip([p for p in live if p >= K], [p for p in range(K) if self.refs[p] == 0]))
        to = dict(moves)
        refs = [0] * self.pages
        for p in live:
            refs[to.get(p, p)] = self.refs[p]
        self.refs = refs
        for b, row in enumerate(self.table):
            held = pages_of(self.lens[b], self.P)
            self.table[b] = [to.get(p, p) if i < held else -1 for i, p in enumerate(row)]
        return moves + [(-1, -1)] * (self.pages // 2 - len(moves))
