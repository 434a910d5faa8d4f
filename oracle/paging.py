"""Serving over the paged 8-bit cache: the tables of a step from the requests'
lengths, and the choice of pages by a score of their keys' bounds.

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


def page_bounds(values, scale):
    """Bounds of one page and head: values [tokens, dim] (of the E4M3 codes), its key
    scale.  (codes int [2, dim], step).  NaN is left out, and 0 where there is nothing else."""
    hi, lo = np.nan_to_num(np.fmax.reduce(values)), np.nan_to_num(np.fmin.reduce(values))
    top = max(np.abs(hi).max(), np.abs(lo).max())
    if top == 0:
        return np.zeros((2, values.shape[1]), dtype=np.int64), np.float32(0)
    codes = np.rint(np.stack([hi, lo]) * 127 / top).astype(np.int64)      # (float64: exact but for the division)
    return codes, np.float32(np.float32(top * float(scale)) / np.float32(127))


def query_codes(q):
    """(codes int [heads, dim], units float32 [heads]) of queries [heads, dim]; the unit of a
    head that is not finite is NaN."""
    whole = np.isfinite(q).all(axis=1)
    q = np.where(whole[:, None], q, 0.0)
    top = np.abs(q).max(axis=1, keepdims=True)
    codes = np.rint(q * 127 / np.where(top > 0, top, 1)).astype(np.int64)
    return codes, np.where(whole, top[:, 0].astype(np.float32) / np.float32(127), np.float32(np.nan))


def page_score(codes, units, bounds, step):
    """Score of a page for a key head's queries: codes int [heads, dim], bounds int [2, dim].
    (No comparison with NaN holds: heads that are not finite are passed over.)"""
    best = -np.inf
    for i, unit in zip(codes, units):
        total = int(np.maximum(i * bounds[0], i * bounds[1]).sum())
        value = np.float32(float(total) * float(unit))
        best = value if value > best else best
    return np.float32(float(best) * float(step))


def choose(scores, seen, count, first, recent):
    """Pages taken of 0 .. seen - 1, ascending; scores[j] of page j (None: not in the cache; NaN
    counts as -infinity)."""
    scores = [s if s is None or s == s else -np.inf for s in scores]
    if seen <= count:
        return list(range(seen))
    middle = range(first, seen - recent)
    best = sorted(middle, key=lambda j: (scores[j] is None, 0 if scores[j] is None else -scores[j], j))
    return sorted(list(range(first)) + best[:count - first - recent] + list(range(seen - recent, seen)))
