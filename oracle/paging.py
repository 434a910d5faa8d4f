"""Serving over the paged 8-bit cache: the tables of a step from the requests'
lengths.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain Python and numpy.

Readings: tokens are dropped and pages given back before any is taken; pages are
taken from the pool's end, in the order in which they stand there; from the first
sequence for which pages or rows are missing on, none gets rows.
"""

import numpy as np


class Pool:
    """Sequences (rows of page numbers, tokens held) and the stack of free pages."""

    def __init__(self, table, kv_len, stack, count, page_size):
        self.table = [list(map(int, r)) for r in table]
        self.kv_len, self.stack = list(map(int, kv_len)), list(map(int, stack))
        self.count, self.page = int(count), page_size
        self.width = len(self.table[0]) if self.table else 0

    def pages(self, tokens):
        return -(-tokens // self.page)

    def step(self, new, drop, kept, rows):
        """(cu_rows, positions, slots) of a step; the state changes in place."""
        n, most = len(self.kv_len), self.width * self.page
        count = min(max(self.count, 0), len(self.stack))
        for b in range(n):
            held = min(max(self.kv_len[b], 0), most)
            base = max(held - max(drop[b], 0), 0)
            for entry in range(self.pages(max(base, min(max(kept[b], 0), held))), self.pages(held)):
                if count < len(self.stack):
                    self.stack[count] = self.table[b][entry]
                    count += 1
            self.kv_len[b] = base
        cu, taken, full = [0], [], False
        for b in range(n):
            base, want = self.kv_len[b], max(new[b], 0)
            if base + want > most:
                want = 0
            entries = range(self.pages(base), self.pages(base + want))
            full = full or len(taken) + len(entries) > count or cu[-1] + want > rows
            if not full:
                taken += [(b, e) for e in entries]
            cu.append(cu[-1] + (0 if full else want))
        self.count = count - len(taken)
        for i, (b, e) in enumerate(taken):
            self.table[b][e] = self.stack[self.count + i]
        positions, slots = [], []
        for b in range(n):
            for t in range(self.kv_len[b], self.kv_len[b] + cu[b + 1] - cu[b]):
                page = self.table[b][t // self.page]
                positions.append(t)
                slots.append(page * self.page + t % self.page if 0 <= page < len(self.stack) else -1)
            self.kv_len[b] += cu[b + 1] - cu[b]
        return np.array(cu), np.array(positions, dtype=np.int64), np.array(slots, dtype=np.int64)
