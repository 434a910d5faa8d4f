"""Pins of the attention oracle's cache: rows of several sequences, a page's scale
over several steps, and exactly which codes a growing scale touches."""

import numpy as np

from oracle import attention as OA


def _value(cache, kind, page, slot, e=0):
    return OA.E4M3_VALUES[cache.codes[kind][page, 0, slot, e]] * cache.scale[kind][page, 0]


def _cache(pages=4):
    codes = [np.full((pages, 1, 16, 64), c, dtype=np.uint8) for c in (0x38, 0x40)]       # 1 and 2
    return OA.Cache(codes[0], codes[1], np.full((pages, 1), 4.0), np.full((pages, 1), 8.0))


def test_rows_go_to_their_own_sequences():
    c = _cache()
    x = np.zeros((6, 1, 64))
    x[:, 0, 0] = [1, 2, 4, 8, 16, 32]
    c.append(np.array([[1], [3], [0]]), [0, 2, 0], [3, 0, 3], x, -2 * x)
    assert [_value(c, 0, 1, s) for s in range(3)] == [1, 2, 4] and [_value(c, 0, 0, s) for s in range(3)] == [8, 16, 32]
    assert [_value(c, 1, 1, s) for s in range(3)] == [-2, -4, -8] and [_value(c, 1, 0, s) for s in range(3)] == [-16, -32, -64]
    assert c.scale[0][1, 0] == 2.0 ** -6 and c.scale[0][0, 0] == 2.0 ** -3        # 4 <= 448 s, 32 <= 448 s
    assert np.all(c.codes[0][[2, 3]] == 0x38) and c.scale[0][3, 0] == 4.0         # pages of no one


def test_a_smaller_token_keeps_the_held_scale():
    c = _cache()
    x = np.zeros((1, 1, 64))
    x[0, 0, 0] = 400.0
    c.append(np.array([[2]]), [0], [1], x, x)
    held = c.codes[0][2, 0, 0].copy()
    c.append(np.array([[2]]), [1], [1], x / 256, x / 256)
    assert c.scale[0][2, 0] == c.scale[1][2, 0] == 1.0
    assert np.array_equal(c.codes[0][2, 0, 0], held) and _value(c, 0, 2, 1) == 1.5       # (1.5625 is halfway to 1.625)


def test_growth_touches_the_slots_in_front_and_no_other():
    c = _cache()
    x = np.zeros((2, 1, 64))
    x[:, 0, 0] = 448 * 8.0                                      # keys from 4 to 8, values keep 8
    c.append(np.array([[1]]), [5], [2], x, x)
    assert c.scale[0][1, 0] == 8.0 and c.scale[1][1, 0] == 8.0
    assert np.all(c.codes[0][1, 0, :5] == 0x30)                 # 1 became 1 / 2: slots 0 .. 4, all elements
    assert np.all(c.codes[0][1, 0, 5:7, 0] == 0x7E) and np.all(c.codes[0][1, 0, 5:7, 1:] == 0)
    assert np.all(c.codes[0][1, 0, 7:] == 0x38)                 # behind: as they were, whatever they now mean
    assert np.all(c.codes[1][1, 0, :5] == 0x40) and np.all(c.codes[1][1, 0, 7:] == 0x40)
