"""Refusals and arguments of the Python layer of the attention.  CPU only: what
passes the checks stops at tensors that are not on the GPU."""

import pytest
import torch

from paper_2609_04098_amd import attention as A
from tests.test_attention_abi import _tensors

BF16 = torch.bfloat16


def test_tensors_that_require_a_gradient_are_refused():
    c, b, x = _tensors()
    learned, gamma = x.clone().requires_grad_(), torch.ones(64, dtype=BF16, requires_grad=True)
    calls = [lambda: A.qk_norm_rope(learned, None), lambda: A.qk_norm_rope(None, learned), lambda: A.qk_norm_rope(x, learned),
             lambda: A.qk_norm_rope(x, None, q_gamma=gamma), lambda: A.qk_norm_rope(x, x, k_gamma=gamma),
             lambda: A.qk_norm_rope(x, None, q_out=learned), lambda: A.kv_append(c, b, learned, x),
             lambda: A.kv_append(c, b, x, learned), lambda: A.kv_append(c, b, x, x, gamma),
             lambda: A.attention(learned, c, b), lambda: A.attention(x, c, b, out=learned),
             lambda: A.attention(learned * 2, c, b)]                # (not a leaf)
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="gradient"):
        A.KVCache(c.k, c.v, c.k_scale.clone().requires_grad_(), c.v_scale, 16)
    # tensors that require none pass with gradients on
    with pytest.raises(ValueError, match="GPU"):
        A.attention(x, c, b)


def test_a_single_page_has_any_stride():
    buf, s = torch.zeros(4 * 16 * 64, dtype=torch.uint8), torch.zeros(8)
    odd = [torch.as_strided(buf, (1, 2, 16 * 64), (stride, 16 * 64, 1)) for stride in (0, 7)]
    c = A.KVCache(*odd, torch.as_strided(s, (1, 2), (0, 1)), torch.as_strided(s, (1, 2), (5, 1)), 16)
    assert (c.struct.k_page_stride, c.struct.v_page_stride, c.struct.scale_page_stride) == (2048, 2048, 2)
    assert c.struct.num_pages == 1
    two = torch.as_strided(buf, (2, 1, 16 * 64), (2048, 16 * 64, 1))
    with pytest.raises(ValueError, match="v_scale"):                # of two pages they do
        A.KVCache(two, two, torch.zeros(2, 1), torch.as_strided(s, (2, 1), (4, 1)), 16)


def test_calibrated_scales_of_keys_and_of_values():
    c = A.alloc_kv_cache(3, 2, 64, 16, "cpu", scale=(0.25, 0.5))
    assert (c.k_scale == 0.25).all() and (c.v_scale == 0.5).all()
    c = A.alloc_kv_cache(3, 2, 64, 16, "cpu", scale=0.125)
    assert (c.k_scale == 0.125).all() and (c.v_scale == 0.125).all()
    c = A.alloc_kv_cache(3, 2, 64, 16, "cpu")
    assert not c.k_scale.any() and not c.v_scale.any()
    with pytest.raises(ValueError, match="scale"):
        A.alloc_kv_cache(3, 2, 64, 16, "cpu", scale=(0.25, 0.5, 1.0))
