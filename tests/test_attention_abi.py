"""The attention entry points are exported, match their header, and refuse
invalid arguments synchronously, before any HIP call (these paths need no GPU);
the Python layer refuses wrong tensors."""

import ctypes
import os
import re

import pytest
import torch

from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import nvfp4 as C
from paper_2609_04098_amd import nvfp4_attention as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "nvfp4_attention.h")
FAKE = 0x100000   # 16-byte aligned, never dereferenced: validation fails first


def test_header_matches_the_binding_and_the_library():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(nvfp4_[a-z0-9_]+)\s*\(", text))) == sorted(N.SIGNATURES)
    for name in N.SIGNATURES:
        assert hasattr(N.lib(), name)
    for struct, fields in (("nvfp4_kv_cache", N.KvCacheStruct), ("nvfp4_kv_batch", N.KvBatchStruct)):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
        assert re.findall(r"(\w+);", body) == [f[0] for f in fields._fields_]


def _norm_rope(**kw):
    a = dict(q=FAKE, ldq=512, hq=4, gq=FAKE, qo=FAKE + 4096, ldqo=512, k=FAKE, ldk=128, hk=1, gk=None, ko=FAKE + 8192,
             ldko=128, rows=3, dim=128, eps=1e-6, pos=FAKE, freq=FAKE, rot=128, inter=0)
    a.update(kw)
    return N.lib().nvfp4_qk_norm_rope(a["q"], a["ldq"], a["hq"], a["gq"], a["qo"], a["ldqo"], a["k"], a["ldk"], a["hk"],
                                      a["gk"], a["ko"], a["ldko"], a["rows"], a["dim"], a["eps"], a["pos"], a["freq"],
                                      a["rot"], a["inter"], None)


@pytest.mark.parametrize("bad", [
    dict(dim=96), dict(dim=0), dict(rows=-1), dict(rows=1 << 24), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(rot=8), dict(rot=144), dict(rot=-16), dict(inter=2), dict(pos=None), dict(freq=None),
    dict(pos=FAKE + 2), dict(freq=FAKE + 1), dict(q=None), dict(q=FAKE + 8), dict(qo=None), dict(ldq=504), dict(ldq=516),
    dict(ldq=1 << 31), dict(hq=-1), dict(hq=1025, ldq=1 << 20, ldqo=1 << 20), dict(gq=FAKE + 4), dict(gk=FAKE + 2),
    dict(ldk=120), dict(ko=FAKE + 2), dict(ldko=64), dict(qo=FAKE, ldqo=520)])
def test_norm_rope_refuses(bad):
    assert _norm_rope(**bad) == C.NVFP4_EINVAL


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, num_pages=4, page_size=32, kv_heads=2, head_dim=128,
             k_page_stride=8192, v_page_stride=8192, scale_page_stride=2)
    a.update(kw)
    return N.KvCacheStruct(**a)


def _batch(**kw):
    a = dict(page_table=FAKE, kv_len=FAKE, cu_rows=FAKE, page_table_stride=8, max_pages=8, n_seqs=3, rows=5,
             max_kv_len=256)
    a.update(kw)
    return N.KvBatchStruct(**a)


def _append(cache=None, batch=None, **kw):
    a = dict(k=FAKE, ldk=256, v=FAKE, ldv=256, gamma=None, eps=0.0, pos=None, freq=FAKE, rot=64, inter=1, mode=0)
    a.update(kw)
    c, b = cache if cache is not None else _cache(), batch if batch is not None else _batch()
    return N.lib().nvfp4_kv_append(ctypes.byref(c), ctypes.byref(b), a["k"], a["ldk"], a["v"], a["ldv"], a["gamma"],
                                   a["eps"], a["pos"], a["freq"], a["rot"], a["inter"], a["mode"], None)


def _attend(cache=None, batch=None, **kw):
    a = dict(q=FAKE, ldq=512, hq=4, y=FAKE, ldy=512, lse=None, scale=0.1, causal=1, window=0, ws=None, wsb=0)
    a.update(kw)
    c, b = cache if cache is not None else _cache(), batch if batch is not None else _batch()
    return N.lib().nvfp4_kv_attention(ctypes.byref(c), ctypes.byref(b), a["q"], a["ldq"], a["hq"], a["y"], a["ldy"],
                                      a["lse"], a["scale"], a["causal"], a["window"], a["ws"], a["wsb"], None)


BAD_CACHES = [
    dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=FAKE + 8), dict(v=FAKE + 1),
    dict(k_scale=FAKE + 2), dict(v_scale=FAKE + 1), dict(num_pages=0), dict(num_pages=1 << 31), dict(page_size=8),
    dict(page_size=48), dict(page_size=256, head_dim=64), dict(page_size=128, head_dim=256, k_page_stride=1 << 20,
                                                               v_page_stride=1 << 20), dict(kv_heads=0),
    dict(head_dim=96), dict(k_page_stride=8176), dict(v_page_stride=8184), dict(v_page_stride=8200),
    dict(scale_page_stride=1)]
BAD_BATCHES = [
    dict(page_table=None), dict(kv_len=None), dict(page_table=FAKE + 2), dict(kv_len=FAKE + 1), dict(cu_rows=FAKE + 2),
    dict(cu_rows=None), dict(page_table_stride=7), dict(max_pages=-1), dict(max_pages=1 << 26, page_table_stride=1 << 26),
    dict(n_seqs=-1), dict(n_seqs=1 << 24), dict(rows=-1), dict(rows=1 << 24), dict(max_kv_len=-1)]


@pytest.mark.parametrize("call", [_append, _attend])
@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_refused(call, bad):
    assert call(cache=_cache(**bad)) == C.NVFP4_EINVAL
    assert N.lib().nvfp4_kv_attention_workspace(ctypes.byref(_cache(**bad)), ctypes.byref(_batch()), 4) == 0


@pytest.mark.parametrize("call", [_append, _attend])
@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_batches_refused(call, bad):
    assert call(batch=_batch(**bad)) == C.NVFP4_EINVAL
    assert N.lib().nvfp4_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_batch(**bad)), 4) == 0


def test_null_structures_are_refused():
    f = N.lib()
    assert f.nvfp4_kv_append(None, ctypes.byref(_batch()), FAKE, 256, FAKE, 256, None, 0.0, None, None, 0, 0, 0,
                             None) == C.NVFP4_EINVAL
    assert f.nvfp4_kv_attention(ctypes.byref(_cache()), None, FAKE, 512, 4, FAKE, 512, None, 0.1, 1, 0, None, 0,
                                None) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(mode=2), dict(mode=-1), dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(ldk=248),
    dict(ldv=260), dict(gamma=FAKE + 2), dict(eps=-1e-9), dict(pos=FAKE + 2), dict(freq=None), dict(rot=24),
    dict(rot=256), dict(inter=3)])
def test_append_refuses(bad):
    assert _append(**bad) == C.NVFP4_EINVAL


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(y=None), dict(q=FAKE + 2), dict(y=FAKE + 4), dict(ldq=504), dict(ldy=516), dict(hq=3), dict(hq=0),
    dict(hq=1026, ldq=1 << 20, ldy=1 << 20), dict(lse=FAKE + 2), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(scale=3e38), dict(causal=2), dict(window=-1), dict(window=1 << 31)])
def test_attention_refuses(bad):
    assert _attend(**bad) == C.NVFP4_EINVAL


def test_attention_refuses_more_rows_than_it_counts():
    c = _cache()
    b = _batch(rows=(1 << 24) - 1)
    assert _attend(cache=c, batch=b, hq=130, ldq=1 << 15, ldy=1 << 15) == C.NVFP4_EINVAL


def test_attention_wants_its_workspace():
    c, b = _cache(num_pages=4096), _batch(cu_rows=None, n_seqs=1, rows=1, max_pages=4096, page_table_stride=4096,
                                          max_kv_len=131072)
    need = N.lib().nvfp4_kv_attention_workspace(ctypes.byref(c), ctypes.byref(b), 4)
    assert need > 0
    assert _attend(cache=c, batch=b) == C.NVFP4_EINVAL
    assert _attend(cache=c, batch=b, ws=FAKE + 8, wsb=need) == C.NVFP4_EINVAL
    assert _attend(cache=c, batch=b, ws=FAKE, wsb=need - 1) == C.NVFP4_EWORKSPACE
    short = _batch(cu_rows=None, n_seqs=1, rows=1, max_pages=4096, page_table_stride=4096, max_kv_len=100)
    assert N.lib().nvfp4_kv_attention_workspace(ctypes.byref(c), ctypes.byref(short), 4) == 0


def _tensors():
    c = A.alloc_kv_cache(4, 2, 64, 16, "cpu")
    b = A.Batch(torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    return c, b, torch.zeros(3, 2, 64, dtype=torch.bfloat16)


def test_python_layer_refuses_wrong_tensors():
    c, b, x = _tensors()
    rope = A.Rope(torch.zeros(32))
    pos = torch.zeros(3, dtype=torch.int32)
    bad = [
        lambda: A.Rope(torch.zeros(12)), lambda: A.Rope(torch.zeros(8).double()), lambda: A.Rope(torch.zeros(2, 8)),
        lambda: A.Rope(torch.zeros(8, requires_grad=True)),
        lambda: A.qk_norm_rope(None, None), lambda: A.qk_norm_rope(x, x[:2]), lambda: A.qk_norm_rope(x.float(), None),
        lambda: A.qk_norm_rope(x, None, None, rope), lambda: A.qk_norm_rope(x, None, pos.long(), rope),
        lambda: A.qk_norm_rope(x, None, pos[:2], rope), lambda: A.qk_norm_rope(x.transpose(0, 1), None),
        lambda: A.qk_norm_rope(x, None, q_gamma=torch.ones(64)), lambda: A.qk_norm_rope(x, None, q_out=x[:, :1]),
        lambda: A.Batch(b.page_table.long(), b.kv_len), lambda: A.Batch(b.page_table, b.kv_len[:2]),
        lambda: A.Batch(b.page_table, b.kv_len, rows=4), lambda: A.Batch(b.page_table, b.kv_len, b.kv_len),
        lambda: A.Batch(b.page_table, b.kv_len, torch.zeros(4, dtype=torch.int32)),
        lambda: A.Batch(b.page_table.t(), torch.zeros(2, dtype=torch.int32)),
        lambda: A.KVCache(c.k, c.v[:3], c.k_scale, c.v_scale, 16),
        lambda: A.KVCache(c.k, c.v, c.k_scale.double(), c.v_scale, 16),
        lambda: A.KVCache(c.k, c.v, c.k_scale[:, :1], c.v_scale, 16),
        lambda: A.KVCache(c.k.transpose(1, 2), c.v.transpose(1, 2), c.k_scale, c.v_scale, 2),
        lambda: A.kv_append(c, b, x[:, :1], x), lambda: A.kv_append(c, b, x, x[:2]),
        lambda: A.kv_append(c, b, x, x, positions=pos.long()), lambda: A.kv_append(c, b, x, x, torch.ones(64)),
        lambda: A.attention(x[:2], c, b), lambda: A.attention(torch.zeros(3, 3, 64, dtype=torch.bfloat16), c, b),
        lambda: A.attention(x, c, b, out=x[:, :1]), lambda: A.attention(x.float(), c, b),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    # CPU tensors are refused, not computed
    for call in (lambda: A.qk_norm_rope(x, None), lambda: A.kv_append(c, b, x, x), lambda: A.attention(x, c, b)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_struct_of_strided_buffers():
    pool = torch.zeros(6, 2, 2, 16 * 64, dtype=torch.uint8)          # pages of keys and values side by side
    s = torch.zeros(6, 2, 2)
    c = A.KVCache(pool[:, 0], pool[:, 1], s[:, 0], s[:, 1], 16)
    assert (c.struct.k_page_stride, c.struct.v_page_stride, c.struct.scale_page_stride) == (4096, 4096, 4)
    assert (c.struct.num_pages, c.struct.page_size, c.struct.kv_heads, c.struct.head_dim) == (6, 16, 2, 64)
    assert c.struct.v - c.struct.k == 2048


def test_python_layer_refuses_several_devices():
    c, b, x = _tensors()
    rope, pos, gamma = A.Rope(torch.zeros(32)), torch.zeros(3, dtype=torch.int32), torch.ones(64, dtype=torch.bfloat16)
    far = [t.to("meta") for t in (x, pos, gamma)]
    far_rope = A.Rope(torch.zeros(32, device="meta"))
    for call in (lambda: A.qk_norm_rope(x, far[0]), lambda: A.qk_norm_rope(x, None, far[1], rope),
                 lambda: A.qk_norm_rope(x, None, pos, far_rope), lambda: A.qk_norm_rope(x, x, q_gamma=gamma, k_gamma=far[2]),
                 lambda: A.qk_norm_rope(x, None, q_out=far[0]), lambda: A.kv_append(c, b, x, far[0]),
                 lambda: A.kv_append(c, b, x, x, far[2]), lambda: A.kv_append(c, b, x, x, gamma, rope=far_rope),
                 lambda: A.kv_append(c, b, x, x, gamma, rope=rope, positions=far[1]), lambda: A.attention(far[0], c, b),
                 lambda: A.attention(x, c, b, out=far[0]), lambda: A.attention(x, c, b, workspace=far[0]),
                 lambda: A.Batch(b.page_table, far[1]), lambda: A.Batch(b.page_table.to("meta"), b.kv_len),
                 lambda: A.Batch(b.page_table, b.kv_len, torch.zeros(4, dtype=torch.int32, device="meta"), rows=3),
                 lambda: A.KVCache(c.k, c.v, c.k_scale, c.v_scale.to("meta"), 16)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_a_single_row_has_any_stride():
    x = torch.zeros(640, dtype=torch.bfloat16)
    for t in (x[:128].view(2, 64)[None], torch.as_strided(x, (1, 2, 64), (3, 64, 1)), x[:128].view(1, 2, 64)):
        assert A._rows(t, "q") == (1, 2, 64, 128)
    assert A._rows(torch.as_strided(x, (2, 2, 64), (256, 64, 1)), "q") == (2, 2, 64, 256)
