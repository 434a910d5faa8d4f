"""GPU tests of the choice of pages where queries are not finite.  Everything is equal to
the oracle's, as in test_gpu_selected_attention.py, whose helpers these are."""

import numpy as np
import pytest
import torch

from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import paging as P
from tests import test_gpu_attention as G
from tests import test_gpu_selected_attention as S
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


# 40 and 700 pages: one launch, and two.  Over 16 query heads: more than one product's columns.
@pytest.mark.parametrize("width", [40, 700])
@pytest.mark.parametrize("dim,heads,group", [(64, 2, 1), (64, 1, 17), (128, 2, 5), (128, 1, 40), (256, 1, 3), (256, 1, 33)])
def test_queries_that_are_not_finite(dim, heads, group, width):
    """Such a query head has no say; where all of a key head's are such, pages tie."""
    log("not finite %s" % ((dim, heads, group, width),))
    gen = torch.Generator().manual_seed(dim + group + width)
    n_pages, page, rows = 60, 16, 7
    cache = G._random_cache(gen, n_pages, heads, page, dim, nan=False)
    bounds = S._all_bounds(cache)
    table = torch.randint(-3, n_pages, (rows, width), generator=gen, dtype=torch.int32)      # (some are not there)
    q = G._bf16(gen, rows, heads * group, dim).cuda()
    last = heads * group - 1
    q[1, 0, 3] = NAN
    q[2, last, dim - 1] = INF
    q[3, last // 2, 5], q[3, last // 2, 6] = -INF, INF
    q[4, :, 7] = NAN                                             # none is left
    q[5, :min(16, last), 1] = INF                                # none of the first 16, where there are more
    q[6, 1:, 2] = -INF
    lens = [width * page - 3 * r for r in range(rows)]
    batch = A.Batch(table.cuda(), S._i32(lens))
    needs = P._p.kv_select_pages_workspace(cache.ref, batch.ref)
    assert (needs > 0) == (width > 256)
    for count, first in ((2, 0), (9, 1), (width - 1, 1)):
        sel = P.select_pages(q, cache, batch, bounds, count, first)
        want = S._want_choice(q, cache, bounds, table, lens, [1] * rows, count, first, 1, True)
        S._check_choice(sel, want, cache, table, [1] * rows, count)
        again = P.select_pages(q, cache, batch, bounds, count, first)
        assert torch.equal(sel.index, again.index) and torch.equal(sel.pages, again.pages)
