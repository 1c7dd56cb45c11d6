"""Integer definition of pages that sequences share, from include/iwdft.h's description: one sequence, one page at a time.  CPU only, in place on numpy arrays."""
from __future__ import annotations

import numpy as np


def _pages(n, P):
    return -(-int(n) // P)


class Tables:
    """table [batch, max_pages], lens [batch], free [1 + pages], refs [pages]."""

    def __init__(self, batch, max_pages, n_pages, P, order=None):
        self.P = P
        self.table, self.lens = np.full((batch, max_pages), -1, np.int32), np.zeros(batch, np.int32)
        self.free = np.concatenate([[n_pages], np.arange(n_pages) if order is None else order]).astype(np.int32)
        self.refs = np.zeros(n_pages, np.int32)

    def arrays(self):
        return dict(table=self.table, lens=self.lens, free=self.free, refs=self.refs)

    def copy(self):
        t = Tables.__new__(Tables)
        t.P = self.P
        for k, v in self.arrays().items():
            setattr(t, k, v.copy())
        return t

    def push(self, page):
        self.free[0] += 1
        self.free[self.free[0]] = page

    def pop(self):
        page = int(self.free[self.free[0]])
        self.free[0] -= 1
        self.refs[page] += 1
        return page

    def release(self, page):
        self.refs[page] -= 1
        if self.refs[page] == 0:
            self.push(page)

    def pages(self, b):
        return self.table[b, :_pages(self.lens[b], self.P)].tolist()

    def consistent(self):
        """Every page is either held, as often as it is counted, or free."""
        held = np.zeros_like(self.refs)
        for b in range(len(self.lens)):
            assert len(set(self.pages(b))) == len(self.pages(b))
            for j, p in enumerate(self.pages(b)):
                held[p] += 1
                assert all(p not in self.pages(c) or self.pages(c)[j] == p for c in range(b))
        stack = self.free[1:1 + self.free[0]].tolist()
        return np.array_equal(held, self.refs) and sorted(stack) == np.flatnonzero(held == 0).tolist()

    def fork(self, parent, keep=None):
        B = len(self.lens)
        parent = [int(p) if 0 <= p < B else b for b, p in enumerate(parent)]
        old = [self.pages(b) for b in range(B)]
        lens = [int(self.lens[p]) if keep is None or keep[b] < 0 else min(int(keep[b]), int(self.lens[p])) for b, p in enumerate(parent)]
        new = [old[p][:_pages(n, self.P)] for p, n in zip(parent, lens)]
        for b in range(B):
            for j, p in enumerate(new[b]):
                if j >= len(old[b]) or old[b][j] != p:
                    self.refs[p] += 1
        for b in reversed(range(B)):
            for j in reversed(range(len(old[b]))):
                if j >= len(new[b]) or new[b][j] != old[b][j]:
                    self.release(old[b][j])
        for b in range(B):
            self.table[b, :len(new[b])] = new[b]
            self.lens[b] = lens[b]

    def resize(self, want, n_slots):
        """starts, slots, copies."""
        B, W = self.table.shape
        P, have = self.P, [int(n) for n in self.lens]
        want = [h if w < 0 or w > W * P else int(w) for h, w in zip(have, want)]
        for b in reversed(range(B)):
            for j in reversed(range(_pages(want[b], P), _pages(have[b], P))):
                self.release(int(self.table[b, j]))
            self.lens[b] = min(have[b], want[b])
        there, asked, fresh = int(self.free[0]), 0, 0
        starts, slots, copies = [0], [], np.full((B, 2), -1, np.int32)
        for b in range(B):
            if want[b] > have[b]:
                had, get = _pages(have[b], P), _pages(want[b], P)
                shared = have[b] % P != 0 and self.refs[self.table[b, had - 1]] > 1
                # all that share it leave it in this call, and those before this one have: it is this one's now
                mine = have[b] % P != 0 and any(copies[c, 0] == self.table[b, had - 1] for c in range(b))
                need, new = get - had + int(shared), want[b] - have[b]
                asked, fresh = asked + need, fresh + new
                if fresh <= n_slots and ((need == 0 and not mine) or asked <= there):
                    if shared:
                        page = int(self.table[b, had - 1])
                        self.refs[page] -= 1
                        self.table[b, had - 1] = self.pop()
                        copies[b] = page, self.table[b, had - 1]
                    for j in range(had, get):
                        self.table[b, j] = self.pop()
                    slots += [int(self.table[b, n // P]) * P + n % P for n in range(have[b], want[b])]
                    self.lens[b] = want[b]
            starts.append(len(slots))
        return np.array(starts, np.int32), np.array(slots + [-1] * (n_slots - len(slots)), np.int32), copies

    def compact(self, n_moves):
        n_pages = len(self.refs)
        moves = np.full((n_moves, 2), -1, np.int32)
        to = {}
        for i in range(n_moves):
            held, free = np.flatnonzero(self.refs > 0), np.flatnonzero(self.refs == 0)
            if not len(held) or not len(free) or free[0] > held[-1]:
                break
            moves[i] = held[-1], free[0]
            to[int(held[-1])] = int(free[0])
            self.refs[free[0]], self.refs[held[-1]] = self.refs[held[-1]], 0
        for b in range(len(self.lens)):
            for j in range(_pages(self.lens[b], self.P)):
                self.table[b, j] = to.get(int(self.table[b, j]), self.table[b, j])
        empty = np.flatnonzero(self.refs == 0)[::-1]
        self.free[0], self.free[1:1 + len(empty)] = len(empty), empty
        return moves
