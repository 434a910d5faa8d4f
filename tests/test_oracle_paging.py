"""Pins of the paging oracle (oracle/paging.py): what must hold of any step's tables,
worked examples, and a tally by sets.  CPU only."""

import random
from fractions import Fraction

import numpy as np
import pytest

from oracle import attention as OA
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


def _brute(q, keys):
    return max(float(a @ b) for a in q for b in keys)


@pytest.mark.parametrize("seed", range(4))
def test_bounds_bound_and_round_as_stated(seed):
    rng = np.random.default_rng(seed)
    dim, tokens, heads = 64, 16, 3
    grid = np.array([v for v in OA.E4M3_VALUES if not np.isnan(v)])
    values, scale = rng.choice(grid[np.abs(grid) < 20], (tokens, dim)), 2.0 ** -5
    codes, step = OP.page_bounds(values, scale)
    top = np.abs(values).max()
    assert np.abs(codes).max() == 127 and step == np.float32(np.float32(top * scale) / np.float32(127))
    for e in range(dim):                                   # exact roundings, by rationals
        for row, v in ((0, values[:, e].max()), (1, values[:, e].min())):
            assert codes[row, e] == round(Fraction(float(v)) * 127 / Fraction(float(top)))
    q = rng.standard_normal((heads, dim)).astype(np.float16).astype(np.float64)
    i, units = OP.query_codes(q)
    for a in range(heads):
        most = np.abs(q[a]).max()
        assert [round(Fraction(float(x)) * 127 / Fraction(float(most))) for x in q[a]] == list(i[a])
        assert units[a] == np.float32(np.float32(most) / np.float32(127))
    # The score bounds every product, but for half a step of either factor.
    score = float(OP.page_score(i, units, codes, step))
    slack = max(float(units[a]) * np.abs(codes).max() * float(step) * dim / 2 + float(step) / 2 * np.abs(q[a]).sum()
                for a in range(heads))
    assert score >= _brute(q, values * scale) - slack
    # and is the product itself where a page holds one key, written out.
    one, unit = OP.page_bounds(values[:1].repeat(tokens, 0), scale)
    assert OP.page_score(i[:1], units[:1], one, unit) == np.float32(
        float(np.float32(float(i[0] @ one[0]) * float(units[0]))) * float(unit))
    assert (OP.page_bounds(np.zeros((tokens, dim)), 1.0)[0] == 0).all() and OP.page_bounds(np.zeros((2, 4)), 1.0)[1] == 0
    assert (OP.query_codes(np.zeros((1, 8)))[0] == 0).all()


def test_choice():
    s = [9.0, 1.0, 5.0, 5.0, 7.0, 5.0, None, 0.0]
    assert OP.choose(s, 8, 8, 1, 1) == list(range(8)) and OP.choose(s, 3, 4, 1, 1) == [0, 1, 2]
    assert OP.choose(s, 8, 4, 0, 1) == [0, 2, 4, 7]        # the lowest among equals
    assert OP.choose(s, 8, 5, 1, 2) == [0, 2, 4, 6, 7]
    assert OP.choose(s, 8, 3, 2, 1) == [0, 1, 7] and OP.choose(s, 8, 7, 0, 1) == [0, 1, 2, 3, 4, 5, 7]
    assert OP.choose([-1.0, -3.0, -2.0, 0.0], 4, 3, 0, 1) == [0, 2, 3] and OP.choose(s, 0, 3, 1, 1) == []


def test_a_full_row_and_those_behind_one_that_is_not_served():
    p = _fresh(1, 2, 4)
    assert list(p.step([32], [0], [0], 32)[0]) == [0, 32] and p.count == 2      # all that its row of pages holds
    p = _fresh(3, 4, 3)
    assert list(p.step([16, 48, 1], [0] * 3, [0] * 3, 100)[0]) == [0, 16, 16, 16]      # the last one would have fitted
    assert p.kv_len == [16, 0, 0] and p.count == 2


def test_bounds_of_negative_keys_and_a_choice_of_few():
    codes, step = OP.page_bounds(np.array([[-4.0, 1.0], [-2.0, 2.0]]), 0.5)
    assert codes.tolist() == [[round(-2 * 127 / 4), round(2 * 127 / 4)], [-127, round(127 / 4)]]
    assert step == np.float32(2) / np.float32(127)
    # Two query heads: the larger product counts, whichever comes first.
    i, units = np.array([[127, 0], [0, 127]]), np.array([1.0, 1.0], dtype=np.float32)
    bounds = np.array([[10, 30], [10, 30]])
    assert OP.page_score(i, units, bounds, 1.0) == OP.page_score(i[::-1], units, bounds, 1.0) == 30 * 127
    assert OP.choose([1.0, 2.0], 2, 3, 2, 1) == [0, 1]


def test_queries_that_are_not_finite_have_no_say():
    rng = np.random.default_rng(5)
    q = rng.standard_normal((4, 8))
    bounds = np.array([[9, 4, 3, 8, 1, 7, 2, 5], [-3, -9, -1, 0, -4, 1, -2, -8]])
    i, units = OP.query_codes(q)
    for bad in (np.nan, np.inf, -np.inf):
        some = q.copy()
        some[0, 3] = some[2, 0] = bad
        codes, unit = OP.query_codes(some)
        assert np.isnan(unit[[0, 2]]).all() and (unit[[1, 3]] == units[[1, 3]]).all() and (codes[[1, 3]] == i[[1, 3]]).all()
        assert OP.page_score(codes, unit, bounds, 0.5) == OP.page_score(i[[1, 3]], units[[1, 3]], bounds, 0.5)
        assert np.isneginf(OP.page_score(codes[[0, 2]], unit[[0, 2]], bounds, 0.5))
    # NaN counts as -infinity: behind every number, in front of pages that are not there.
    s = [np.nan, -9.0, None, -np.inf, np.nan, 4.0, 0.0]
    assert OP.choose(s, 7, 3, 0, 1) == [1, 5, 6] and OP.choose(s, 7, 5, 0, 1) == [0, 1, 3, 5, 6]
    assert OP.choose(s, 7, 6, 0, 1) == [0, 1, 3, 4, 5, 6]


def test_bounds_of_keys_that_are_not_numbers():
    nan = np.nan
    values = np.array([[nan, 2.0, nan, -1.0], [3.0, nan, nan, -4.0], [-1.0, nan, nan, nan]])
    codes, step = OP.page_bounds(values, 0.5)
    assert codes.tolist() == [[round(3 * 127 / 4), round(2 * 127 / 4), 0, round(-127 / 4)],
                              [round(-127 / 4), round(2 * 127 / 4), 0, -127]] and step == np.float32(2) / np.float32(127)
    codes, step = OP.page_bounds(values[:, 2:3], 0.5)
    assert not codes.any() and step == 0
