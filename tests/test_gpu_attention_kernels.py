"""GPU tests of every kernel of the attention, each by a step that takes it: under a
causal mask, without one, with a window, with value scales that are no powers of two,
behind an attention sink.  Comparison and tolerances: those of test_gpu_attention_precision.py."""

import numpy as np
import pytest
import torch

from paper_2609_04098_amd import attention as A
from tests import test_gpu_attention_precision as P
from tests.attention_forms import EVERY, name, names
from tests.gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("step", EVERY, ids=name)
def test_every_kernel(step):
    dim, page, heads, group, lens, counts = step[:6]
    log("every kernel %s" % name(step))
    case = P.Case(dim, page, heads, lens, seed=dim + lens[0])
    q = P._queries(case, sum(counts), heads * group)
    assert _of(case, counts, heads * group) == names(step)
    P._run(case, q, counts)
    P._run(case, q, counts, causal=False)
    # Windows that every row but the first of a new sequence fills, over and within a tile (what a window divides is another plan).
    for window in (17, 64, 500):
        P._run(case, q, counts, window=window)


@pytest.mark.parametrize("step", EVERY, ids=name)
def test_every_kernel_with_scales_that_are_no_powers_of_two(step):
    dim, page, heads, group, lens, counts = step[:6]
    log("every kernel, scales %s" % name(step))
    case = P.Case(dim, page, heads, lens, seed=dim + lens[0] + 1)
    for s in (case.ks, case.vs):
        s *= 0.6 + torch.rand(s.shape, generator=case.gen, device="cuda")
    P._run(case, P._queries(case, sum(counts), heads * group), counts)
    case.ks.fill_(0.013), case.vs.fill_(0.17)                        # one calibrated scale for the tensor
    P._run(case, P._queries(case, sum(counts), heads * group), counts)


@pytest.mark.parametrize("step", [s for s in EVERY if min(n for n in s[4] if n) > 10], ids=name)
def test_a_sink_in_every_kernel(step):
    """One token with values of zero, 18 and 20 nats above all others."""
    dim, page, heads, group, lens, counts = step[:6]
    for nats in (18, 20):
        log("every kernel, sink %s" % name(step))
        case = P.Case(dim, page, heads, lens, seed=dim + lens[0] + nats)
        q = P.add_sink(case, heads * group, counts, nats, 0.3)
        P._run(case, q, counts, scale=1.0)


@pytest.mark.parametrize("step", EVERY, ids=name)
def test_what_lies_in_front_of_a_window_in_every_kernel(step):
    """Infinite and NaN scales of pages that no row sees: y as with others."""
    dim, page, heads, group, lens, counts = step[:6]
    log("every kernel, window %s" % name(step))
    case = P.Case(dim, page, heads, lens, seed=dim + lens[0] + 2)
    q = P._queries(case, sum(counts), heads * group)
    batch = A.Batch(case.table.int(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda"), rows=sum(counts))
    for window in (3, 1000):
        want = A.attention(q, case.cache(), batch, window=window, return_lse=True)
        clean = case.cache()
        dirty = A.KVCache(clean.k, clean.v, clean.k_scale.clone(), clean.v_scale.clone(), page)
        for b, n in enumerate(lens):
            hidden = case.table[b, :max(0, n - counts[b] - window + 1) // page]
            for i, bad in enumerate((float("inf"), float("nan"))):
                dirty.v_scale[hidden[i::2]], dirty.k_scale[hidden[i::2]] = bad, bad
        got = A.attention(q, dirty, batch, window=window, return_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), window


def _of(case, counts, q_heads):
    lens = torch.tensor(case.lens, dtype=torch.int32, device="cuda")
    cu = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
    return A.attention_kernels(q_heads, case.cache(), A.Batch(case.table.int(), lens, cu, rows=sum(counts)))
