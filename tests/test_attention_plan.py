"""What the host decides about a step of the attention (csrc/attention_plan.h):
steps that one launch cannot hold are refused before any HIP call, and the GPU tests'
steps take the kernels that these tests mean.  CPU only."""

import ctypes

import pytest

from paper_2609_04098_amd import nvfp4 as C
from paper_2609_04098_amd import nvfp4_attention as N
from tests import test_gpu_attention_forms as forms
from tests.attention_forms import EVERY, JOIN, ROWS, TILE, name, names
from tests.test_attention_abi import _append, _attend, _batch, _cache


def _step(n, heads, dim, rows=None, page=16):
    c = _cache(kv_heads=heads, head_dim=dim, page_size=page, k_page_stride=heads * page * dim,
               v_page_stride=heads * page * dim, scale_page_stride=heads)
    return c, _batch(n_seqs=n, rows=n if rows is None else rows, **({"cu_rows": None} if rows is None else {}))


@pytest.mark.parametrize("n,heads,group", [(1 << 21, 8, 5), (1 << 22, 8, 5), ((1 << 24) - 1, 2, 1), (1 << 20, 16, 16),
                                           (1 << 20, 8, 33), (1 << 14, 1024, 1)])
def test_attention_refuses_more_workgroups_than_a_launch_holds(n, heads, group):
    c, b = _step(n, heads, 128)
    assert _attend(c, b, hq=heads * group, ldq=heads * group * 128, ldy=heads * group * 128) == C.NVFP4_EINVAL
    assert N.lib().nvfp4_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), heads * group) == 0


@pytest.mark.parametrize("n,heads,dim,rows,page", [
    (1 << 23, 4, 128, None, 16), (1 << 22, 8, 128, None, 16), (1 << 21, 16, 128, 1 << 23, 16),
    ((1 << 24) - 1, 2, 256, None, 16), (1 << 14, 1024, 256, None, 16), (3 << 20, 8, 128, (1 << 24) - 1, 128)])
def test_append_refuses_more_workgroups_than_a_launch_holds(n, heads, dim, rows, page):
    c, b = _step(n, heads, dim, rows, page)
    assert _append(c, b, ldk=heads * dim, ldv=heads * dim) == C.NVFP4_EINVAL


def _kernels(dim, page, heads, group, lens, rows, window=0, max_len=None, **kw):
    """The kernels of a step whose tables are as wide as its longest sequence wants."""
    width = max(1, max(-(-n // page) for n in lens))
    c = _cache(page_size=page, head_dim=dim, kv_heads=heads, k_page_stride=heads * page * dim,
               v_page_stride=heads * page * dim, scale_page_stride=heads)
    b = _batch(n_seqs=len(lens), rows=rows, max_pages=width, page_table_stride=width,
               max_kv_len=width * page if max_len is None else max_len, **kw)
    got = [N.kv_attention_kernel(ctypes.byref(c), ctypes.byref(b), heads * group, window, part) for part in (0, 1)]
    assert (got[1] is None) or N.lib().nvfp4_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), heads * group) > 0
    return [k for k in got if k is not None]


@pytest.mark.parametrize("step", EVERY, ids=name)
def test_steps_reach_the_kernels_that_they_name(step):
    assert _kernels(*step[:5], sum(step[5])) == names(step)


def test_every_kernel_has_a_step():
    got = {k for step in EVERY for k in names(step)}
    want = {k % d for d in (64, 128, 256) for k in
            [ROWS + "1,4,false>", ROWS + "1,4,true>", ROWS + "1,8,false>", ROWS + "2,4,false>", ROWS + "2,4,true>",
             TILE + "false>", TILE + "true>"] + [JOIN + "%d,%d>" % (t, s) for t in (1, 2, 8) for s in (1, 4)]}
    assert got == want and len(got) == 39


@pytest.mark.parametrize("case", [c for c in forms.TILES if c[0] != 64], ids=lambda c: "d%d_p%d_h%dx%d" % c[:4])
def test_the_gpu_tests_of_128_rows_take_128(case):
    """(Rows: five behind the last sequence.  Heads of 64: EVERY's.)"""
    for window in (0, 50, 130, 1):
        assert _kernels(*case[:5], sum(case[5]) + 5, window)[0].startswith(TILE % case[0])


@pytest.mark.parametrize("dim,hkv,group,lens,counts", [
    (256, 8, 8, [2000, 1300, 50, 1999], [60, 40, 50, 50]), (256, 32, 2, [1500, 700], [65, 65]), (128, 1, 8, [60000], [8187]),
    (64, 1, 8, [16000], [8187])])
def test_the_gpu_tests_of_128_rows_in_pieces_take_both(dim, hkv, group, lens, counts):
    got = _kernels(dim, 64, hkv, group, lens, sum(counts) + 5)
    assert got[0] == TILE % dim + "true>" and got[1].startswith(JOIN % dim + "8,")


@pytest.mark.parametrize("dim,longest,full", [(64, 599, 330), (64, 600, 850), (64, 9999, 850), (64, 1 << 20, 500), (128, 599, 150),
                                              (128, 600, 400), (128, 1599, 400), (128, 1600, 480), (256, 3499, 65),
                                              (256, 3500, 24)])
def test_where_tiles_of_128_rows_begin(dim, longest, full):
    for heads, group in ((1, 128), (4, 32), (2, 64)):
        rows = full * 128 // (heads * group)
        for n, tile in ((rows, TILE), (rows - 1, ROWS)):
            assert _kernels(dim, 16, heads, group, [longest], n, max_len=longest)[0].startswith(tile % dim)
    # never for sequences of up to 64 packed rows
    assert _kernels(dim, 16, 8, 4, [longest] * 1000, 16000, max_len=longest)[0].startswith(ROWS % dim)


def test_the_kernel_query():
    c, b = _cache(), _batch()
    f = lambda c=c, b=b, hq=4, window=0, part=0: N.lib().nvfp4_kv_attention_kernel(
        None if c is None else ctypes.byref(c), None if b is None else ctypes.byref(b), hq, window, part)
    assert f() == b"kv_attention_rows_kernel<128,1,8,false>" and f(part=1) is None
    for bad in (dict(c=None), dict(b=None), dict(hq=3), dict(window=-1), dict(window=1 << 31), dict(part=2), dict(part=-1),
                dict(b=_batch(rows=0)), dict(b=_batch(n_seqs=0)), dict(c=_cache(head_dim=96))):
        assert f(**bad) is None
    # the largest steps that one launch holds, and the next ones
    for n, heads, group, fits in (((1 << 21) - 1, 8, 5, True), (1 << 21, 8, 5, False), (3355443, 5, 1, True),
                                  ((1 << 20) - 1, 16, 16, True), (1 << 20, 8, 17, True), (1 << 20, 8, 33, False)):
        c, b = _step(n, heads, 128)
        assert (f(c, b, heads * group) is not None) == fits
