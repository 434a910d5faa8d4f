"""What the host decides about a step of the attention (csrc/attention_plan.h):
steps that one launch cannot hold are refused before any HIP call.  CPU only."""

import ctypes

import pytest

from paper_2609_04098_amd import nvfp4 as C
from paper_2609_04098_amd import nvfp4_attention as N
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
