"""Pins of the paging oracle (oracle/paging.py): what must hold of any step's tables,
worked examples, and a tally by sets.  CPU only."""

import random

import pytest

from oracle import paging as OP


def _fresh(n, width, pages, page=16):
    return OP.Pool([[-7] * width for _ in range(n)], [0] * n, range(pages), pages, page)


def test_worked_example():
    p = _fresh(3, 4, 8)
    cu, pos, slots = p.step([17, 0, 16], [0] * 3, [0] * 3, 40)
    assert list(cu) == [0, 17, 17, 33] and p.kv_len == [17, 0, 16] and p.count == 5
    assert p.table[0][:2] == [5, 6] and p.table[2][0] == 7          # the pool's end, in its order
    assert list(pos) == list(range(17)) + list(range(16))
    assert slots[0] == 5 * 16 and slots[16] == 6 * 16 and slots[17] == 7 * 16
    cu, pos, slots = p.step([1, 1, 1], [2, 0, 16], [0] * 3, 3)       # 17 - 2 + 1: its second page goes back
    assert p.kv_len == [16, 1, 1] and list(pos) == [15, 0, 0]
    assert p.table[1][0] == 6 and p.table[2][0] == 7 and p.count == 5      # two given back, two taken


def test_who_is_served():
    p = _fresh(4, 2, 3)
    cu, _, _ = p.step([16, 33, 20, 1], [0] * 4, [0] * 4, 100)        # 33 tokens: no row of 2 pages holds them
    assert list(cu) == [0, 16, 16, 36, 36] and p.count == 0          # no page is left for the last one
    cu, _, _ = p.step([1, 0, 0, 1], [16, 0, 0, 0], [0] * 4, 1)
    assert list(cu) == [0, 1, 1, 1, 1] and p.kv_len == [1, 0, 20, 0]      # no row is left for it
    cu, _, _ = p.step([0, 0, 0, 1], [5, 0, 100, 0], [0, 0, 16, 0], 1)
    assert p.kv_len == [0, 0, 0, 1] and p.count == 1                 # its first page is kept


@pytest.mark.parametrize("seed", range(6))
def test_every_page_is_in_one_place(seed):
    rng = random.Random(seed)
    n, width, pages, page = rng.randint(1, 9), rng.randint(1, 6), rng.randint(3, 30), rng.choice([16, 32])
    p = _fresh(n, width, pages, page)
    for _ in range(30):
        before = [list(r) for r in p.table], list(p.kv_len)
        new = [rng.choice([0, 1, 1, 5, rng.randint(0, width * page)]) for _ in range(n)]
        drop = [rng.choice([0, 0, 1, 7, 1000]) for _ in range(n)]
        rows = rng.randint(0, 2 * width * page)
        cu, pos, slots = p.step(new, drop, [0] * n, rows)
        used = [p.table[b][e] for b in range(n) for e in range(p.pages(p.kv_len[b]))]
        assert sorted(used + p.stack[:p.count]) == list(range(pages))
        assert cu[-1] == len(pos) == len(slots) <= rows and len(set(slots)) == len(slots)
        for b in range(n):
            base = max(before[1][b] - drop[b], 0)
            got = cu[b + 1] - cu[b]
            assert got in (0, new[b]) and p.kv_len[b] == base + got
            assert p.table[b][:p.pages(base)] == before[0][b][:p.pages(base)]      # held tokens stay where they are
            assert list(pos[cu[b]:cu[b + 1]]) == list(range(base, base + got))
