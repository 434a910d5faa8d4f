"""The paging entry points are exported, match their header, and refuse invalid
arguments synchronously, before any HIP call (these paths need no GPU); the Python
layer refuses wrong tensors."""

import ctypes
import os
import re

import pytest
import torch

from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import nvfp4 as C
from paper_2609_04098_amd import nvfp4_paging as N
from paper_2609_04098_amd import paging as P
from tests.test_attention_abi import BAD_BATCHES, BAD_CACHES, FAKE, ROOT, _batch, _cache

HEADER = os.path.join(ROOT, "include", "nvfp4_paging.h")
STRUCTS = {"nvfp4_requests": N.RequestsStruct, "nvfp4_shared_prefix": N.SharedPrefixStruct,
           "nvfp4_kv_bounds": N.BoundsStruct}


def test_header_matches_the_binding_and_the_library():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(nvfp4_[a-z0-9_]+)\s*\(", text))) == sorted(N.SIGNATURES)
    for name in N.SIGNATURES:
        assert hasattr(N.lib(), name)
    assert set(re.findall(r"typedef struct (\w+)", text)) == set(STRUCTS)
    for struct, fields in STRUCTS.items():
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
        assert re.findall(r"(\w+);", body) == [f[0] for f in fields._fields_]


def _requests(**kw):
    a = dict(page_table=FAKE, kv_len=FAKE, free_pages=FAKE, free_count=FAKE, page_table_stride=8, max_pages=8, n_seqs=3,
             num_pages=16, page_size=32)
    a.update(kw)
    return N.RequestsStruct(**a)


def _tables(requests=None, **kw):
    a = dict(new=FAKE, drop=None, kept=None, cu=FAKE, pos=FAKE, slots=FAKE, rows=5, ws=FAKE, wsb=1 << 20)
    a.update(kw)
    r = requests if requests is not None else _requests()
    return N.lib().nvfp4_step_tables(ctypes.byref(r), a["new"], a["drop"], a["kept"], a["cu"], a["pos"], a["slots"],
                                     a["rows"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad", [
    dict(page_table=None), dict(kv_len=None), dict(free_pages=None), dict(free_count=None), dict(page_table=FAKE + 2),
    dict(kv_len=FAKE + 1), dict(free_pages=FAKE + 2), dict(free_count=FAKE + 3), dict(page_table_stride=7),
    dict(max_pages=-1), dict(max_pages=1 << 26, page_table_stride=1 << 26), dict(n_seqs=-1), dict(n_seqs=1 << 24),
    dict(num_pages=0), dict(num_pages=1 << 31), dict(page_size=8), dict(page_size=48), dict(page_size=256)])
def test_requests_refused(bad):
    assert _tables(_requests(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(new=None), dict(new=FAKE + 2), dict(drop=FAKE + 1), dict(kept=FAKE + 2), dict(cu=None), dict(cu=FAKE + 2),
    dict(pos=FAKE + 2), dict(slots=FAKE + 4), dict(rows=-1), dict(rows=1 << 24), dict(ws=None), dict(ws=FAKE + 4)])
def test_tables_refuse(bad):
    assert _tables(**bad) == C.NVFP4_EINVAL


def test_tables_want_their_workspace():
    need = N.lib().nvfp4_step_tables_workspace(3)
    assert need > 0 and N.lib().nvfp4_step_tables_workspace(-1) == 0 == N.lib().nvfp4_step_tables_workspace(1 << 24)
    assert _tables(wsb=need - 1) == C.NVFP4_EWORKSPACE
    assert N.lib().nvfp4_step_tables(None, FAKE, None, None, FAKE, None, None, 1, FAKE, 1 << 20, None) == C.NVFP4_EINVAL


def _groups(**kw):
    a = dict(cu_seqs=FAKE, prefix=FAKE, n_groups=2, max_prefix=2000, max_own=60)
    a.update(kw)
    return N.SharedPrefixStruct(**a)


def _long(**kw):
    """A batch whose prefixes may be long enough to be shared."""
    return _batch(**{**dict(max_pages=100, page_table_stride=100, max_kv_len=3200), **kw})


def _attend(cache=None, batch=None, groups=None, **kw):
    a = dict(q=FAKE, ldq=512, hq=4, y=FAKE, ldy=512, lse=None, scale=0.1, causal=1, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    c, b, g = (x if x is not None else f() for x, f in ((cache, _cache), (batch, _long), (groups, _groups)))
    return N.lib().nvfp4_kv_attention_shared(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), a["q"], a["ldq"], a["hq"],
                                             a["y"], a["ldy"], a["lse"], a["scale"], a["causal"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_shared_attention_refuses_caches(bad):
    assert _attend(_cache(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_shared_attention_refuses_batches(bad):
    assert _attend(batch=_batch(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [dict(cu_seqs=None), dict(prefix=None), dict(cu_seqs=FAKE + 2), dict(prefix=FAKE + 1),
                                 dict(n_groups=-1), dict(n_groups=4), dict(max_prefix=-1), dict(max_own=-1)])
def test_shared_attention_refuses_groups(bad):
    assert _attend(groups=_groups(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(y=None), dict(q=FAKE + 2), dict(y=FAKE + 4), dict(ldq=504), dict(ldy=516), dict(hq=3), dict(hq=0),
    dict(hq=1026, ldq=1 << 20, ldy=1 << 20), dict(lse=FAKE + 2), dict(scale=float("nan")), dict(scale=3e38), dict(causal=2),
    dict(ws=None), dict(ws=FAKE + 8)])
def test_shared_attention_refuses(bad):
    assert _attend(**bad) == C.NVFP4_EINVAL


def test_shared_attention_wants_its_workspace():
    f, c, b, g = N.lib(), _cache(), _long(), _groups()
    need = f.nvfp4_kv_attention_shared_workspace(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), 4)
    assert need > 0 and _attend(wsb=need - 1) == C.NVFP4_EWORKSPACE
    assert f.nvfp4_kv_attention_shared_workspace(ctypes.byref(c), ctypes.byref(b), ctypes.byref(_groups(n_groups=9)), 4) == 0
    assert f.nvfp4_kv_attention_shared_workspace(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), 3) == 0
    for null in range(3):
        args = [ctypes.byref(c), ctypes.byref(b), ctypes.byref(g)]
        args[null] = None
        assert f.nvfp4_kv_attention_shared(*args, FAKE, 512, 4, FAKE, 512, None, 0.1, 1, FAKE, 1 << 30, None) == C.NVFP4_EINVAL


def _kernels(cache, batch, groups, heads):
    f = N.lib().nvfp4_kv_attention_shared_kernel
    return [f(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(groups), heads, part) for part in (0, 1)]


def test_which_steps_share():
    """By their sizes: prefixes of 1536 tokens, fewer than 64 rows of a sequence."""
    c = _cache()
    rows = lambda n, r: _long(n_seqs=n, rows=r)
    share = lambda k: k[0].startswith(b"kv_attention_shared_kernel<128,") and k[1].startswith(b"kv_attention_shared_join_kernel<128,")
    assert share(_kernels(c, rows(3, 5), _groups(max_prefix=1536), 4))
    assert not share(_kernels(c, rows(3, 5), _groups(max_prefix=1535), 4))
    assert share(_kernels(c, rows(4, 124), _groups(), 4)) and not share(_kernels(c, rows(4, 128), _groups(), 4))
    assert not share(_kernels(c, rows(4, 4), _groups(n_groups=0), 4))
    assert not share(_kernels(c, _batch(), _groups(), 4))                    # (256 tokens are all that its table holds)
    assert _kernels(c, rows(3, 5), _groups(n_groups=5), 4) == _kernels(c, rows(3, 0), _groups(), 4) == [None, None]
    f = N.lib().nvfp4_kv_attention_shared_kernel
    assert f(ctypes.byref(c), ctypes.byref(_long()), ctypes.byref(_groups()), 4, 2) is None


@pytest.mark.parametrize("n,heads,group", [(1 << 21, 8, 5), ((1 << 24) - 1, 2, 1), (1 << 20, 8, 33)])
def test_shared_attention_refuses_more_workgroups_than_a_launch_holds(n, heads, group):
    c = _cache(kv_heads=heads, page_size=16, k_page_stride=heads * 2048, v_page_stride=heads * 2048, scale_page_stride=heads)
    b = _long(n_seqs=n, rows=n, cu_rows=None)
    assert _attend(c, b, hq=heads * group, ldq=heads * group * 128, ldy=heads * group * 128) == C.NVFP4_EINVAL


def test_shared_attention_refuses_wrong_tensors():
    c = A.alloc_kv_cache(4, 2, 64, 16, "cpu")
    b = A.Batch(_i32(3, 2), _i32(3))
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    g = P.SharedPrefix(_i32(3), _i32(2))
    for call in (lambda: P.SharedPrefix(_i32(2), _i32(2)), lambda: P.SharedPrefix(_i32(3).long(), _i32(2)),
                 lambda: P.SharedPrefix(_i32(3), _i32(2).float()), lambda: P.SharedPrefix(_i32(6)[::2], _i32(2)),
                 lambda: P.shared_attention(x[:2], c, b, g), lambda: P.shared_attention(x.float(), c, b, g),
                 lambda: P.shared_attention(x[:, :3], c, b, g), lambda: P.shared_attention(x, c, b, g, out=x[:, :2]),
                 lambda: P.shared_attention(x, c, b, P.SharedPrefix(_i32(5), _i32(4))),
                 lambda: P.shared_attention(x.requires_grad_(), c, b, g)):
        with pytest.raises(ValueError):
            call()
    x = x.detach()
    far = x.to("meta")
    for call in (lambda: P.SharedPrefix(_i32(3).to("meta"), _i32(2)), lambda: P.shared_attention(far, c, b, g),
                 lambda: P.shared_attention(x, c, b, g, out=far), lambda: P.shared_attention(x, c, b, g, workspace=far)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="GPU"):
        P.shared_attention(x, c, b, g)


def _bounds(**kw):
    a = dict(codes=FAKE, step=FAKE, page_stride=512, step_stride=2)
    a.update(kw)
    return N.BoundsStruct(**a)


def _page_bounds(cache=None, batch=None, bounds=None):
    c, b, g = (x if x is not None else f() for x, f in ((cache, _cache), (batch, _batch), (bounds, _bounds)))
    return N.lib().nvfp4_kv_page_bounds(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), None)


def _far(**kw):
    """A batch of few rows and long sequences, whose scores take a workspace."""
    return _batch(**{**dict(max_pages=1000, page_table_stride=1000, max_kv_len=32000), **kw})


def _select(cache=None, batch=None, bounds=None, **kw):
    a = dict(q=FAKE, ldq=512, hq=4, count=4, first=1, recent=1, causal=1, index=FAKE, pages=FAKE, tokens=FAKE, ws=FAKE,
             wsb=1 << 30)
    a.update(kw)
    c, b, g = (x if x is not None else f() for x, f in ((cache, _cache), (batch, _far), (bounds, _bounds)))
    return N.lib().nvfp4_kv_select_pages(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), a["q"], a["ldq"], a["hq"],
                                         a["count"], a["first"], a["recent"], a["causal"], a["index"], a["pages"],
                                         a["tokens"], a["ws"], a["wsb"], None)


def _selected(cache=None, **kw):
    a = dict(q=FAKE, ldq=512, hq=4, rows=5, count=4, pages=FAKE, tokens=FAKE, y=FAKE, ldy=512, lse=None, scale=0.1, ws=FAKE,
             wsb=1 << 30)
    a.update(kw)
    c = cache if cache is not None else _cache()
    return N.lib().nvfp4_kv_attention_selected(ctypes.byref(c), a["q"], a["ldq"], a["hq"], a["rows"], a["count"], a["pages"],
                                               a["tokens"], a["y"], a["ldy"], a["lse"], a["scale"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("call", [_page_bounds, _select, _selected])
@pytest.mark.parametrize("bad", BAD_CACHES)
def test_selection_refuses_caches(call, bad):
    assert call(cache=_cache(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("call", [_page_bounds, _select])
@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_selection_refuses_batches(call, bad):
    assert call(batch=_batch(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("call", [_page_bounds, _select])
@pytest.mark.parametrize("bad", [dict(codes=None), dict(step=None), dict(codes=FAKE + 8), dict(step=FAKE + 2),
                                 dict(page_stride=496), dict(page_stride=520), dict(step_stride=1),
                                 dict(page_stride=1 << 31), dict(step_stride=1 << 31)])
def test_selection_refuses_bounds(call, bad):
    assert call(bounds=_bounds(**bad)) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=FAKE + 2), dict(ldq=504), dict(hq=3), dict(hq=0), dict(count=0), dict(count=(1 << 25) + 1),
    dict(first=-1), dict(recent=0), dict(first=4), dict(first=2, recent=3), dict(recent=5), dict(causal=2),
    dict(first=(1 << 63) - 1), dict(recent=(1 << 63) - 1), dict(index=None), dict(pages=None), dict(tokens=None),
    dict(index=FAKE + 2), dict(pages=FAKE + 1), dict(tokens=FAKE + 2), dict(ws=None), dict(ws=FAKE + 8)])
def test_select_refuses(bad):
    assert _select(**bad) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(y=None), dict(q=FAKE + 2), dict(y=FAKE + 4), dict(ldq=504), dict(ldy=516), dict(hq=3), dict(hq=0),
    dict(lse=FAKE + 2), dict(scale=float("inf")), dict(rows=-1), dict(rows=1 << 24), dict(count=0), dict(count=(1 << 25) + 1),
    dict(pages=None), dict(tokens=None), dict(pages=FAKE + 2), dict(tokens=FAKE + 1),
    dict(rows=(1 << 24) - 1, hq=130, ldq=1 << 15, ldy=1 << 15)])
def test_selected_attention_refuses(bad):
    assert _selected(**bad) == C.NVFP4_EINVAL


def test_selection_wants_its_workspaces():
    f, c, b = N.lib(), _cache(), _far()
    need = f.nvfp4_kv_select_pages_workspace(ctypes.byref(c), ctypes.byref(b))
    assert need > 0 and _select(wsb=need - 1) == C.NVFP4_EWORKSPACE
    assert f.nvfp4_kv_select_pages_workspace(ctypes.byref(c), ctypes.byref(_batch(rows=-1))) == 0
    assert f.nvfp4_kv_select_pages_workspace(ctypes.byref(c), ctypes.byref(_batch())) == 0      # (one launch)
    need = f.nvfp4_kv_attention_selected_workspace(ctypes.byref(c), 1, 4, 2000)
    assert need > 0 and _selected(rows=1, count=2000, wsb=need - 1) == C.NVFP4_EWORKSPACE
    assert _selected(rows=1, count=2000, ws=None) == C.NVFP4_EINVAL == _selected(rows=1, count=2000, ws=FAKE + 4)
    assert f.nvfp4_kv_attention_selected_workspace(ctypes.byref(c), 1, 4, 0) == 0
    assert f.nvfp4_kv_attention_selected_workspace(ctypes.byref(c), 0, 4, 2000) == 0
    assert f.nvfp4_kv_page_bounds(None, ctypes.byref(b), ctypes.byref(_bounds()), None) == C.NVFP4_EINVAL
    assert _select(batch=_batch(n_seqs=0)) == C.NVFP4_EINVAL      # rows of no sequence


def test_selection_refuses_more_workgroups_than_a_launch_holds():
    heads = 64
    c = _cache(kv_heads=heads, page_size=16, k_page_stride=heads * 2048, v_page_stride=heads * 2048, scale_page_stride=heads)
    b, g = _batch(n_seqs=1 << 21, rows=1 << 21, cu_rows=None), _bounds(page_stride=1 << 16, step_stride=heads)
    assert _page_bounds(c, b, g) == C.NVFP4_EINVAL
    assert _select(c, b, g, hq=heads, ldq=heads * 128, wsb=1 << 62) == C.NVFP4_EINVAL
    assert _selected(c, hq=heads, rows=1 << 21, ldq=heads * 128, ldy=heads * 128) == C.NVFP4_EINVAL


def test_selection_refuses_wrong_tensors():
    c = A.alloc_kv_cache(4, 2, 64, 16, "cpu")
    b = A.Batch(_i32(3, 2), _i32(3))
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    g = P.alloc_page_bounds(c)
    sel = P.Selection(_i32(3, 2, 4), _i32(3, 2, 4), _i32(3))
    other = P.alloc_page_bounds(A.alloc_kv_cache(5, 2, 64, 16, "cpu"))
    for call in (lambda: P.PageBounds(g.codes.float(), g.step), lambda: P.PageBounds(g.codes[:, :1], g.step),
                 lambda: P.PageBounds(g.codes.transpose(1, 2), g.step), lambda: P.PageBounds(g.codes, g.step.double()),
                 lambda: P.PageBounds(g.codes[:1].expand(4, 2, 2, 64), g.step), lambda: P.PageBounds(g.codes, g.step[:1].expand(4, 2)),
                 lambda: P.page_bounds(c, b, other), lambda: P.select_pages(x, c, b, other, 4),
                 lambda: P.select_pages(x[:2], c, b, g, 4), lambda: P.select_pages(x.float(), c, b, g, 4),
                 lambda: P.select_pages(x, c, b, g, 0), lambda: P.select_pages(x, c, b, g, 4, first=4),
                 lambda: P.select_pages(x, c, b, g, 4, recent=0), lambda: P.select_pages(x, c, b, g, 4, first=-1),
                 lambda: P.select_pages(x, c, b, g, 5, out=sel), lambda: P.Selection(_i32(3, 2, 4), _i32(3, 2, 3), _i32(3)),
                 lambda: P.Selection(_i32(3, 2, 4), _i32(3, 2, 4), _i32(2)), lambda: P.Selection(_i32(3, 2, 4).long(), _i32(3, 2, 4), _i32(3)),
                 lambda: P.selected_attention(x[:2], c, sel), lambda: P.selected_attention(x[:, :3], c, sel),
                 lambda: P.selected_attention(x, A.alloc_kv_cache(4, 4, 64, 16, "cpu"), sel),
                 lambda: P.selected_attention(x, c, sel, out=x[:, :2]), lambda: P.selected_attention(x.requires_grad_(), c, sel)):
        with pytest.raises(ValueError):
            call()
    x = x.detach()
    far, far_sel = x.to("meta"), P.Selection(*[t.to("meta") for t in (sel.index, sel.pages, sel.tokens)])
    for call in (lambda: P.PageBounds(g.codes, g.step.to("meta")), lambda: P.select_pages(far, c, b, g, 4),
                 lambda: P.select_pages(x, c, b, g, 4, out=far_sel), lambda: P.selected_attention(x, c, far_sel),
                 lambda: P.selected_attention(far, c, sel), lambda: P.select_pages(x, c, b, g, 4, workspace=far),
                 lambda: P.page_bounds(c, b, P.PageBounds(g.codes.to("meta"), g.step.to("meta"))),
                 lambda: P.Selection(sel.index, sel.pages.to("meta"), sel.tokens)):
        with pytest.raises(ValueError, match="device"):
            call()
    for call in (lambda: P.page_bounds(c, b, g), lambda: P.select_pages(x, c, b, g, 4), lambda: P.selected_attention(x, c, sel)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_requests_refuse_wrong_tensors():
    table, lens, free, count = _i32(3, 4), _i32(3), _i32(9), _i32(1)
    P.Requests(table, lens, free, count, 16)
    for call in (lambda: P.Requests(table.long(), lens, free, count, 16), lambda: P.Requests(table, _i32(2), free, count, 16),
                 lambda: P.Requests(table, lens.long(), free, count, 16), lambda: P.Requests(table, lens, free[::2], count, 16),
                 lambda: P.Requests(table, lens, _i32(0), count, 16), lambda: P.Requests(table, lens, free, _i32(2), 16),
                 lambda: P.Requests(table, lens, free, count, 24), lambda: P.Requests(table.t(), _i32(4), free, count, 16),
                 lambda: P.Requests(_i32(1, 4).expand(3, 4), lens, free, count, 16),
                 lambda: P.Requests(table, _i32(6)[::2], free, count, 16)):
        with pytest.raises(ValueError):
            call()
    for far in range(4):
        args = [table, lens, free, count]
        args[far] = args[far].to("meta")
        with pytest.raises(ValueError, match="device"):
            P.Requests(*args, 16)


def test_step_tables_refuses_wrong_tensors():
    r = P.alloc_requests(3, 4, 20, 16, "cpu")
    assert r.free_pages.tolist() == list(range(19, -1, -1)) and r.free_count.item() == 20
    new = _i32(3)
    step = P.Step(r, 5)
    for call in (lambda: P.step_tables(r, None, 5), lambda: P.step_tables(r, new.long(), 5),
                 lambda: P.step_tables(r, new[:2], 5), lambda: P.step_tables(r, _i32(6)[::2], 5),
                 lambda: P.step_tables(r, new, 5, drop=_i32(4)), lambda: P.step_tables(r, new, 5, kept=new.float()),
                 lambda: P.step_tables(r, new, 4, out=step), lambda: P.step_tables(r, new, 5, max_len=7, out=step),
                 lambda: P.step_tables(P.alloc_requests(3, 4, 20, 16, "cpu"), new, 5, out=step)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="device"):
        P.step_tables(r, new.to("meta"), 5)
    with pytest.raises(ValueError, match="GPU"):      # CPU tensors are refused, not computed
        P.step_tables(r, new, 5)


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="valid arguments, but no memory behind them")
@pytest.mark.parametrize("rows,pages", [((1 << 16) - 1, 8192), ((1 << 15) + 1, 8192), ((1 << 16) - 1, 2048)])
def test_selection_in_one_launch_is_bounded_by_it_alone(rows, pages):
    """Rows x key heads below 2^22 whose scores need no launch of their own are only stopped
    by the missing device."""
    heads = 64
    c = _cache(kv_heads=heads, page_size=16, k_page_stride=heads * 2048, v_page_stride=heads * 2048, scale_page_stride=heads)
    b = _batch(n_seqs=rows, rows=rows, cu_rows=None, max_pages=pages, page_table_stride=pages, max_kv_len=16 * pages)
    g = _bounds(page_stride=1 << 16, step_stride=heads)
    status = _select(c, b, g, hq=heads, ldq=heads * 128, wsb=1 << 62)
    assert status in (C.NVFP4_EUNSUPPORTED, C.NVFP4_EHIP)
    more = _batch(n_seqs=1 << 16, rows=1 << 16, cu_rows=None, max_pages=pages, page_table_stride=pages, max_kv_len=16 * pages)
    assert _select(c, more, g, hq=heads, ldq=heads * 128, wsb=1 << 62) == C.NVFP4_EINVAL
