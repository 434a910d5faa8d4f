"""GPU tests of what the attention must not look at: pages in front of a window,
rows whose tokens would be before the first one, windows and lengths near 2^31."""

import numpy as np
import pytest
import torch

from paper_2609_04098_amd import attention as A
from tests.gpu_common import log
from tests.test_gpu_attention import _check, _cu, _i32, _random_cache

pytestmark = pytest.mark.gpu

FORMS = [      # dim, page, key heads, group, lengths, new rows: 16 rows whole and in pieces, 32, 128, 128 in pieces
    (128, 16, 2, 4, [300, 95], [1, 1]), (64, 16, 2, 4, [9000, 700], [1, 1]), (256, 16, 1, 4, [9000, 333], [2, 1]),
    (128, 16, 1, 7, [200, 90], [60, 30]), (128, 16, 32, 8, [300, 700], [70, 65]), (256, 16, 8, 8, [2000, 1300], [60, 40]),
]


def _name(c):
    return "d%d_h%dx%d_%d" % (c[0], c[2], c[3], c[4][0])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("form", FORMS, ids=_name)
def test_pages_in_front_of_a_window_may_hold_anything(form, causal):
    """Infinite and NaN scales and NaN codes in pages that no row sees: y as with clean ones."""
    dim, page, hkv, group, lens, counts = form
    gen = torch.Generator().manual_seed(dim + lens[0])
    width = -(-max(lens) // page)
    table = torch.randperm(len(lens) * width, generator=gen).view(len(lens), width)
    cache = _random_cache(gen, len(lens) * width, hkv, page, dim, nan=False)
    q = torch.randn(sum(counts), hkv * group, dim, generator=gen).to(torch.bfloat16).cuda()
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=sum(counts))
    for window in (3, 40, 100):
        log("front %s window %d" % (form, window))
        want = A.attention(q, cache, batch, causal=causal, window=window, return_lse=True)
        dirty = A.KVCache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone(), page)
        for b, n in enumerate(lens):
            hidden = table[b, :max(0, n - counts[b] - window + 1) // page].cuda()
            dirty.k[hidden], dirty.v[hidden] = 0x7F, 0xFF
            for i, bad in enumerate((float("inf"), float("nan"), float("-inf"))):
                dirty.v_scale[hidden[i::3]], dirty.k_scale[hidden[i::3]] = bad, bad
        got = A.attention(q, dirty, batch, causal=causal, window=window, return_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), window


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (False, 5), (False, 40)])
@pytest.mark.parametrize("form", [(128, 16, 2, 4, [3, 0, 20], [5, 2, 1]), (64, 32, 1, 3, [50, 7], [70, 9]),
                                  (128, 16, 32, 8, [30, 60], [66, 70]), (256, 32, 32, 2, [70, 40], [75, 60])], ids=_name)
def test_more_new_rows_than_tokens(form, causal, window):
    """Rows whose tokens would be before 0 see nothing under a causal mask, and without one what the formula says."""
    dim, page, hkv, group, lens, counts = form
    log("rows before 0 %s %s %d" % (form, causal, window))
    gen = torch.Generator().manual_seed(dim + window)
    width = max(1, -(-max(lens) // page))
    table = torch.randperm(len(lens) * width, generator=gen).view(len(lens), width)
    cache = _random_cache(gen, len(lens) * width, hkv, page, dim, nan=False)
    q = (torch.randn(sum(counts), hkv * group, dim, generator=gen) * 0.5).to(torch.bfloat16).cuda()
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=sum(counts))
    y, lse = A.attention(q, cache, batch, causal=causal, window=window, return_lse=True)
    _check(y, lse, cache, q, table, lens, counts, dim ** -0.5, causal, window)
    if causal:
        first = [sum(counts[:b]) for b in range(len(counts))]
        for b, r in enumerate(first):
            early = slice(r, r + max(0, counts[b] - lens[b]))
            assert not y[early].any() and torch.isneginf(lse[early]).all()


@pytest.mark.parametrize("window", [2 ** 30 + 40, 2 ** 31 - 130, 2 ** 31 - 1])
@pytest.mark.parametrize("form", [(64, 16, 1, 3, [1], [1, 1, 2]), (128, 16, 32, 8, [1], [66, 70, 5])], ids=_name)
def test_windows_near_the_largest(form, window):
    """Windows over 2^30, for rows of any number up to 2^31 - 2 and for rows before token 0."""
    dim, page, hkv, group, _, counts = form
    gen = torch.Generator().manual_seed(dim)
    table = torch.randperm(24, generator=gen).view(3, 8)
    cache = _random_cache(gen, 24, hkv, page, dim, nan=False)
    q = (torch.randn(sum(counts), hkv * group, dim, generator=gen) * 0.5).to(torch.bfloat16).cuda()
    for lens in ([2 ** 31 - 1, 2 ** 30 + 60, 1], [window + 100 if window + 100 < 2 ** 31 else 90, 2 ** 31 - 3, 0]):
        for causal in (True, False):
            batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=sum(counts))
            y, lse = A.attention(q, cache, batch, causal=causal, window=window, return_lse=True)
            _check(y, lse, cache, q, table, lens, counts, dim ** -0.5, causal, window)
            seen = 2 ** 31 - 1 - window < 128 if lens[0] == 2 ** 31 - 1 else True
            assert bool(y[counts[0] - 1].any()) == seen
