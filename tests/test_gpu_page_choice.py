"""GPU tests of the pages' bounds and of the choice of pages where keys or queries are not
finite.  Everything is equal to
the oracle's, as in test_gpu_selected_attention.py, whose helpers these are."""

import numpy as np
import pytest
import torch

from oracle import attention as OA
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


@pytest.mark.parametrize("dim,page,heads", [(64, 16, 2), (128, 32, 1), (128, 128, 3), (256, 16, 2), (256, 64, 1)])
def test_bounds_of_keys_that_are_not_numbers(dim, page, heads):
    """NaN of both codes: among an element's tokens, all of an element, all of a page."""
    log("NaN keys %s" % ((dim, page, heads),))
    gen = torch.Generator().manual_seed(dim + page)
    n_pages = 8
    cache = G._random_cache(gen, n_pages, heads, page, dim, nan=True)
    places = torch.from_numpy(OA.byte_places(page, dim, False))
    nat = cache.k.cpu()[:, :, places]                             # [page, head, token, element]
    nat[1, :, :, dim // 2] = 0x7F
    nat[2, :, :, 0], nat[2, :, ::2, dim - 1], nat[2, :, 1::2, dim - 1] = 0xFF, 0x7F, 0xFF
    nat[3, 0] = 0x7F
    nat[4, heads - 1, :, 1:] = 0xFF                               # one element is left
    nat[5, :, 1:] = 0x7F                                          # one token is left
    k = torch.empty_like(cache.k.cpu())
    k[:, :, places] = nat
    cache.k.copy_(k)
    table, lens = torch.randperm(n_pages, generator=gen).view(2, 4).int(), [4 * page, 4 * page]
    bounds = P.PageBounds(torch.full((n_pages, heads, 2, dim), -77, dtype=torch.int8, device="cuda"),
                          torch.full((n_pages, heads), -7.0, device="cuda"))
    P.page_bounds(cache, A.Batch(table.cuda(), S._i32(lens), S._i32([0, lens[0], 2 * lens[0]]), rows=2 * lens[0]), bounds)
    want = S._want_bounds(cache, table, lens, lens, np.zeros((n_pages, heads, 2, dim), dtype=np.int64),
                          np.zeros((n_pages, heads), dtype=np.float32))
    assert np.array_equal(bounds.codes.cpu().numpy(), want[0]) and np.array_equal(bounds.step.cpu().numpy(), want[1])
    assert not bounds.codes[3, 0].any() and bounds.step[3, 0] == 0
    q = G._bf16(gen, 2, heads * 2, dim).cuda()
    sel = P.select_pages(q, cache, A.Batch(table.cuda(), S._i32(lens)), bounds, 3)
    S._check_choice(sel, S._want_choice(q, cache, bounds, table, lens, [1, 1], 3, 1, 1, True), cache, table, [1, 1], 3)


@pytest.mark.parametrize("rows,heads,width", [(5, 2, 3000), (20, 3, 9000)])
def test_a_choice_keeps_few_scores(rows, heads, width):
    """Of tables over 256 pages: what a call scores is gone with it, but for a megabyte at
    most, on any stream."""
    log("memory of a choice %s" % ((rows, heads, width),))
    gen = torch.Generator().manual_seed(4)
    n_pages, count = 50, 6
    cache = G._random_cache(gen, n_pages, heads, 16, 64, nan=False)
    bounds = S._all_bounds(cache)
    batch = A.Batch(torch.randint(0, n_pages, (rows, width), generator=gen, dtype=torch.int32).cuda(),
                    S._i32([16 * width - 7 * r for r in range(rows)]))
    q = G._bf16(gen, rows, heads * 3, 64).cuda()
    scores = 4 * rows * heads * width
    assert P._p.kv_select_pages_workspace(cache.ref, batch.ref) == scores
    want = P.select_pages(q, cache, batch, bounds, count)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    others = [P.select_pages(q, cache, batch, bounds, count, stream=side) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    others += [P.select_pages(q, cache, batch, bounds, count, workspace=torch.empty(scores, dtype=torch.uint8, device="cuda")),
               P.select_pages(q, cache, batch, bounds, count, out=P.Selection(want.index.clone(), want.pages.clone(), want.tokens + 1))]
    for sel in [want] + others:
        assert sel.index.untyped_storage().nbytes() <= 4 * (2 * rows * heads * count + rows) + (1 << 20)
        assert torch.equal(sel.index, want.index) and torch.equal(sel.pages, want.pages) and torch.equal(sel.tokens, want.tokens)
