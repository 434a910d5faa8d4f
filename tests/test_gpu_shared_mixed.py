"""GPU tests of the attention with shared prefixes where a prompt's rows stand among single
tokens: in a group, behind its prefix, and in none.  Comparison and tolerances: those of
test_gpu_shared_attention.py, whose steps these are."""

import pytest

from paper_2609_04098_amd import paging as P
from tests import test_gpu_shared_attention as H
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

# dim, page, key heads, group, groups, own tokens, new rows, whether a step of these sizes shares
STEPS = [
    # a prompt of its own behind the groups
    *[(d, 16, 2, 5, [(40, 1600)], [3 + 7 * i for i in range(40)] + [700], [1] * 40 + [200], True) for d in (64, 128, 256)],
    # one that begins behind a group's prefix, as its first, its last and the only sequence that has rows
    *[(d, 32, 1, 4, [(12, 640), (9, 1536)], [300] + [5 + i for i in range(20)], [250] + [1] * 20, True) for d in (64, 128, 256)],
    (128, 32, 2, 8, [(20, 1600)], [2 + i for i in range(19)] + [90], [1] * 19 + [77], True),
    (64, 16, 2, 3, [(5, 1600)], [9, 8, 140, 6, 5], [0, 0, 100, 0, 0], True),
    # one whose rows reach into the prefix beside those that share it
    (128, 16, 2, 2, [(30, 1600)], [20] * 29 + [60], [1] * 29 + [300], True),
    # so many rows that the step's average leaves nothing shared
    (128, 16, 2, 5, [(10, 1600)], [12] * 10 + [900], [1] * 10 + [900], False),
]


@pytest.mark.parametrize("step", STEPS, ids=H._name)
def test_prompts_among_single_tokens(step):
    log("mixed %s" % H._name(step))
    dim, page, heads, group, groups, own, counts, shares = step
    s = H.Step(dim, page, heads, group, groups, own, counts, sum(own) + dim + 1, True)
    tight = dict(max_len=max(1536, max(p for _, p in groups)), max_own=max(own))
    names = P.shared_attention_kernels(s.heads, s.case.cache(), s.batch(max_len=max(s.lens)), s.shared(**tight))
    assert any("shared" in n for n in names) == shares
    s.check(hints=tight, max_len=max(s.lens), pages=True)
    s.check(causal=False, hints=tight, max_len=max(s.lens))
    s.check()
    s.check(hints=dict(max_len=1536, max_own=1), scale=-0.05)
