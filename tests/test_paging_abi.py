"""The paging entry points are exported, match their header, and refuse invalid
arguments synchronously, before any HIP call (these paths need no GPU); the Python
layer refuses wrong tensors."""

import ctypes
import os
import re

import pytest
import torch

from paper_2609_04098_amd import nvfp4 as C
from paper_2609_04098_amd import nvfp4_paging as N
from paper_2609_04098_amd import paging as P
from tests.test_attention_abi import FAKE, ROOT

HEADER = os.path.join(ROOT, "include", "nvfp4_paging.h")
STRUCTS = {"nvfp4_requests": N.RequestsStruct}


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
