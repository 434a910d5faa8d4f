"""GPU tests of the choice of pages over many rounds of a workgroup's scores: tables of 257
to 20000 pages, for each head size in one launch and in two, up to 40 query heads of a key
head.  Bounds are given (any whole numbers), and everything is equal to the oracle's; scores
by whole products of matrices, which test_scores_are_the_oracles compares with it."""

import numpy as np
import pytest
import torch

from oracle import paging as OP
from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import paging as P
from tests.gpu_common import log

PAGE = 16


def _scores(q, codes, step):
    """float32 [pages]: of queries [group, dim], bounds int [pages, 2, dim], step float32 [pages]."""
    i, units = OP.query_codes(q)
    i, codes = i.astype(np.float64), codes.astype(np.float64)      # (whole numbers below 2^53: exact)
    total = np.maximum(i, 0) @ codes[:, 0].T + np.minimum(i, 0) @ codes[:, 1].T
    best = (total * units.astype(np.float64)[:, None]).astype(np.float32).max(axis=0)
    return (best.astype(np.float64) * step.astype(np.float64)).astype(np.float32)


def _some(seed, n_pages, heads, dim, rows, group):
    gen = np.random.default_rng(seed)
    codes = gen.integers(0, 128, (n_pages, heads, 2, dim))
    codes[:, :, 1] *= -1
    step = np.exp2(gen.uniform(-9, -8, (n_pages, heads))).astype(np.float32)
    q = torch.from_numpy(gen.standard_normal((rows, heads * group, dim)).astype(np.float32)).to(torch.bfloat16)
    return gen, codes, step, q


def test_scores_are_the_oracles():
    _, codes, step, q = _some(1, 9, 2, 64, 3, 4)
    for r in range(3):
        for h in range(2):
            x = q[r, 4 * h:4 * h + 4].double().numpy()
            i, units = OP.query_codes(x)
            want = [OP.page_score(i, units, codes[p, h], step[p, h]) for p in range(9)]
            assert np.array_equal(_scores(x, codes[:, h], step[:, h]), np.array(want, dtype=np.float32))


# dim, key heads, group, rows, pages of a table, count, first, recent
ONE = [(64, 8, 2, 32, 800, 60, 20, 1), (128, 4, 5, 64, 2100, 700, 1, 2), (256, 2, 3, 128, 800, 300, 17, 1),
       (128, 16, 20, 16, 257, 100, 0, 1), (256, 4, 17, 64, 1100, 200, 33, 5), (64, 4, 40, 64, 1300, 333, 3, 1),
       (128, 8, 5, 33, 2049, 128, 1, 1), (64, 2, 3, 128, 8192, 500, 1, 1), (256, 8, 2, 40, 2060, 64, 0, 1)]
TWO = [(64, 5, 3, 51, 2100, 600, 1, 1), (128, 3, 5, 85, 2100, 400, 20, 3), (256, 5, 2, 51, 2100, 300, 1, 1),
       (128, 7, 2, 30, 8000, 1000, 1, 2), (64, 4, 2, 15, 20000, 3000, 17, 1), (256, 2, 20, 20, 5000, 900, 1, 1),
       (128, 2, 40, 25, 9000, 64, 0, 1), (256, 1, 3, 60, 20000, 9000, 1, 1), (64, 3, 17, 40, 3000, 100, 2, 1)]


def rounds(c):
    """Rounds that the scoring waves of a workgroup take: 16 pages each, of 16 waves, or of 4
    for their share of the pages."""
    dim, heads, group, rows, width = c[:5]
    if c in ONE:
        return -(-width // 256)
    each = min(16, -(-(rows * heads * -(-width // 64)) // 2048))      # (times 64 pages)
    return min(each, -(-width // 64))


def test_every_head_size_takes_many_rounds_in_both_forms():
    for form in (ONE, TWO):
        for dim in (64, 128, 256):
            mine = [c for c in form if c[0] == dim]
            assert any(rounds(c) >= 4 for c in mine) and any(c[2] > 16 and rounds(c) >= 2 for c in mine), (dim, mine)
        assert any(c[6] > 16 for c in form)


@pytest.mark.gpu
@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("c", ONE + TWO, ids=lambda c: "_".join(str(x) for x in c[:5]))
def test_choice_over_many_rounds(c, drafts):
    dim, heads, group, rows, width, count, first, recent = c
    log("rounds %s %s" % (c, drafts))
    n_pages = 2500
    gen, codes, step, q = _some(sum(c), n_pages, heads, dim, rows, group)
    counts = [1] * rows
    if drafts:      # several rows each, one sequence without any, two rows behind the last one
        counts = [0] + [3] * ((rows - 2) // 3)
        counts[-1] += rows - 2 - sum(counts)
    table = gen.integers(0, n_pages, (len(counts), width))
    table[0, ::7], table[-1, 5::9] = -1, n_pages                     # pages that are not there
    lens = [max(n, width * PAGE - int(gen.integers(0, width * PAGE)) * (i % 3 > 0) - i % PAGE) for i, n in enumerate(counts)]
    cache = A.alloc_kv_cache(n_pages, heads, dim, PAGE, "cuda")
    bounds = P.PageBounds(torch.from_numpy(codes.astype(np.int8)).cuda(), torch.from_numpy(step).cuda())
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    batch = A.Batch(i32(table), i32(lens), i32([0] + list(np.cumsum(counts))) if drafts else None, rows=rows)
    assert (P._p.kv_select_pages_workspace(cache.ref, batch.ref) == 0) == (c in ONE)
    sel = P.select_pages(q.cuda(), cache, batch, bounds, count, first, recent)
    index, pages, tokens = sel.index.cpu().numpy(), sel.pages.cpu().numpy(), sel.tokens.tolist()
    row = 0
    for b, n in enumerate(counts):
        for i in range(n):
            t = lens[b] - n + i
            seen = t // PAGE + 1
            for h in range(heads):
                of = _scores(q[row, h * group:(h + 1) * group].double().numpy(), codes[:, h], step[:, h])
                entries = table[b, :seen]
                there = (entries >= 0) & (entries < n_pages)
                scores = of[np.clip(entries, 0, n_pages - 1)].tolist()
                scores = [s if ok else None for s, ok in zip(scores, there)]
                want = OP.choose(scores, seen, count, first, recent)
                assert index[row, h, :len(want)].tolist() == want, (row, h)
                assert np.array_equal(pages[row, h, :len(want)], table[b, want])
                assert (index[row, h, len(want):] == -1).all() and (pages[row, h, len(want):] == -1).all()
            assert tokens[row] == (min(seen, count) - 1) * PAGE + t % PAGE + 1
            row += 1
    assert tokens[row:] == [-1] * (rows - row)
