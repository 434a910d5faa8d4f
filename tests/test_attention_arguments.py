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
