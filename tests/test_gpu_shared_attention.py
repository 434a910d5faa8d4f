"""GPU tests of the attention with shared prefixes against float64 on the same codes.
Comparison and tolerances: those of test_gpu_attention_precision.py (both parts of a
row keep what those allow of their own largest probability; a join adds roundings that
the sums' 32 of them hold)."""

import numpy as np
import pytest
import torch

from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import paging as P
from tests import test_gpu_attention_precision as T
from tests.gpu_common import log

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Step:
    """Groups [(sequences, prefix)], then `alone` sequences of none; own: tokens of each
    behind its prefix; counts: new rows."""

    def __init__(self, dim, page, heads, group, groups, own, counts, seed, cu=True, least=2048):
        prefix = [p for n, p in groups for _ in range(n)]
        prefix += [0] * (len(own) - len(prefix))
        lens = [p + o for p, o in zip(prefix, own)]
        self.case = T.Case(dim, page, heads, lens, seed)
        self.first = [0] + list(np.cumsum([n for n, _ in groups]))
        for g, (n, p) in enumerate(groups):      # (a page that the prefix fills in part is not shared beyond it)
            for b in range(self.first[g] + 1, self.first[g] + n):
                self.case.table[b, :-(-p // page)] = self.case.table[self.first[g], :-(-p // page)]
        if self.case.table.shape[1] * page < least:      # a table that could hold a prefix worth sharing
            more = least // page - self.case.table.shape[1]
            self.case.table = torch.cat((self.case.table, self.case.table[:, :1].expand(-1, more)), dim=1).contiguous()
        self.counts, self.lens, self.heads = counts, lens, heads * group
        self.groups = groups
        self.q = T._queries(self.case, sum(counts), self.heads)
        self.cu = _i32([0] + list(np.cumsum(counts))) if cu else None

    def shared(self, **kw):
        return P.SharedPrefix(_i32(self.first), _i32([p for _, p in self.groups]), **kw)

    def batch(self, **kw):
        return A.Batch(self.case.table.int(), _i32(self.lens), self.cu, rows=sum(self.counts), **kw)

    def check(self, causal=True, scale=None, hints=None, max_len=None, pages=False):
        scale = self.case.dim ** -0.5 if scale is None else scale
        y, lse = P.shared_attention(self.q, self.case.cache(), self.batch(max_len=max_len), self.shared(**(hints or {})),
                                    scale=scale, causal=causal, return_lse=True)
        T._compare(y, lse, self.case, self.q, self.counts, scale, causal, 0, T._some, pages)
        return y


SHARED, JOIN = "kv_attention_shared_kernel<%d,%s>", "kv_attention_shared_join_kernel<%d,%d>"

# dim, page, key heads, group, groups, own tokens, new rows, row offsets or not, the kernel's rows and the
# waves that join one.  (The host is told of prefixes that are worth sharing.)
STEPS = [
    # one group, single tokens, without row offsets
    *[(d, p, 2, 3, [(4, 96)], [1, 5, 40, 100], [1] * 4, False, ("1,1", 4)) for d, p in ((64, 16), (128, 32), (256, 64))],
    (128, 128, 1, 1, [(2, 128)], [1, 1], [1, 1], False, ("1,1", 4)),
    # many sequences: 32 and 48 packed rows a tile, pieces of the prefix
    *[(d, 32, 2, 5, [(40, 2016)], [3 + 7 * i for i in range(40)], [1] * 40, False, ("1,1", 4)) for d in (64, 128, 256)],
    *[(d, 16, 2, 8, [(50, 512)], [30] * 50, [1] * 50, False, ("1,1", 1)) for d in (64, 128, 256)],
    *[(d, 32, 8, 8, [(100, 1504)], [9 + i for i in range(100)], [1] * 100, False, ("2,1" if d == 64 else "1,1", 1))
      for d in (64, 128, 256)],
    (128, 16, 16, 8, [(45, 6000)], [5 + i for i in range(45)], [1] * 45, False, ("3,1", 1)),
    (128, 16, 16, 16, [(30, 3008), (1, 64), (43, 3200)], [9 + i for i in range(76)], [1] * 76, True, ("3,1", 1)),
    (128, 64, 1, 4, [(5, 9024)], [300, 1, 64, 2, 700], [1] * 5, False, ("1,1", 4)),
    # several groups of all kinds, one without a prefix, sequences of none, some without rows
    (64, 16, 2, 3, [(3, 160), (1, 32), (4, 0), (2, 1600)], [9, 20, 1, 5, 8, 3, 1, 2, 70, 4, 33, 500], [2, 1, 1, 3, 1, 0, 1, 2, 5, 4, 7, 9],
     True, ("1,1", 1)),
    (128, 32, 3, 7, [(2, 64), (0, 96), (3, 640)], [3, 40, 12, 5, 64, 800, 1], [3, 1, 0, 5, 2, 6, 1], True, ("3,2", 4)),
    (64, 32, 3, 7, [(2, 64), (0, 96), (3, 640)], [3, 40, 12, 5, 64, 800, 1], [3, 1, 0, 5, 2, 6, 1], True, ("2,2", 4)),
    (256, 16, 1, 16, [(2, 320), (2, 16)], [10, 20, 11, 2], [4, 3, 5, 2], True, ("8,8", 4)),
    # drafts of many sequences, several rows each behind a common prefix
    *[(d, 32, 4, 4, [(30, 992)], [12 + 5 * i for i in range(30)], [8 + i % 3 for i in range(30)], True,
       ({64: "2,2", 128: "3,2", 256: "8,8"}[d], 1))
      for d in (64, 128, 256)],
    # a prefix that ends inside a page that the sequences share, and inside a tile
    (128, 32, 2, 4, [(3, 75)], [1, 1, 1], [1] * 3, False, ("1,1", 4)),
    # rows of a sequence that fill tiles of their own: computed apart
    (128, 32, 4, 4, [(3, 992)], [500, 320, 77], [500, 320, 70], True, None), (256, 32, 8, 8, [(2, 480)], [90, 80], [70, 66], True, None),
]


def _name(s):
    return "_".join(str(x) for x in s[:4]) + "_" + "_".join("%dx%d" % g for g in s[4])


@pytest.mark.parametrize("step", STEPS, ids=_name)
def test_shared_attention(step):
    log("shared %s" % _name(step))
    dim, page, heads, group, groups, own, counts, cu, form = step
    s = Step(dim, page, heads, group, groups, own, counts, sum(own) + dim, cu, least=2048)
    tight = dict(max_len=max(1536, max(p for _, p in groups)), max_own=max(own))
    names = P.shared_attention_kernels(s.heads, s.case.cache(), s.batch(max_len=max(s.lens)), s.shared(**tight))
    if form is not None:
        assert names == [SHARED % (dim, form[0]), JOIN % (dim, form[1])]
    else:
        assert not any("shared" in n for n in names)
    s.check(hints=tight, max_len=max(s.lens), pages=True)
    s.check(causal=False, hints=tight, max_len=max(s.lens))
    s.check()                                            # nothing known on the host
    s.check(hints=dict(max_len=1536, max_own=1), scale=-0.05)      # too little known
    s.check(hints=dict(max_len=1, max_own=1))            # so little that nothing is shared


def test_every_form_has_a_step():
    got = {(s[0], s[8][0]) for s in STEPS if s[8]}
    assert {(s[0], s[8][1]) for s in STEPS if s[8]} == {(d, j) for d in (64, 128, 256) for j in (1, 4)}
    assert got == {(64, "1,1"), (64, "2,1"), (64, "2,2"), (128, "1,1"), (128, "3,1"), (128, "3,2"), (256, "1,1"), (256, "8,8")}


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_more_groups_than_a_wave_has_lanes(dim):
    log("many groups %d" % dim)
    groups = [(1 + i % 3, 16 * (i % 4)) for i in range(70)]
    n = sum(g for g, _ in groups)
    for cu in (False, True):
        counts = [1] * n if not cu else [i % 3 for i in range(n)]
        s = Step(dim, 16, 1, 2, groups, [1 + counts[i] + i % 20 for i in range(n)], counts, dim, cu)
        s.check(hints=dict(max_len=1536, max_own=25))


@pytest.mark.parametrize("causal", [True, False])
def test_sequences_that_do_not_share(causal):
    """Rows in front of the prefix's end, sequences of nothing and padding in the group:
    each is computed from its own pages, and the group's pages come from one that shares."""
    log("not sharing")
    dim, page = 128, 16
    s = Step(dim, page, 2, 4, [(6, 64)], [5, 9, 3, 40, 1, 0], [2, 3, 1, 2, 1, 0], 11)
    s.lens[0], s.lens[2], s.lens[5] = 0, 40, 0                # nothing; in front of the prefix's end; nothing
    s.counts[0] = 0
    s.q = T._queries(s.case, sum(s.counts), s.heads)
    s.cu = _i32([0] + list(np.cumsum(s.counts)))
    s.case.lens = s.lens
    own = s.case.table.clone()
    own[0], own[5] = 1 << 30, -5                              # their rows of the table may hold anything
    own[2, :3] = own[3, 4:7]                                  # pages of another beginning than the group's
    s.case.table = own
    y = s.check(causal=causal)
    plain = A.attention(s.q, s.case.cache(), s.batch(), causal=causal)
    assert (y.float() - plain.float()).abs().max() <= 2.0 ** -7 * plain.float().abs().max()
    # rows of a sequence that reach into the prefix: all of it is its own
    s.lens[1] = 66
    s.case.lens = s.lens
    s.check(causal=causal)


def test_prefixes_that_make_no_sense():
    """Lengths and offsets out of range are cut; results stay those of attention()."""
    log("no sense")
    s = Step(64, 16, 1, 2, [(3, 48)], [4, 20, 9], [1, 1, 1], 5, False)
    cache, batch = s.case.cache(), s.batch()
    want = A.attention(s.q, cache, batch).float()
    for first, prefix in (([0, 3], [1 << 30]), ([0, 3], [-9]), ([-4, 900], [48]), ([5, 5], [48]), ([3, 0], [48]), ([1, 2], [48]),
                          ([0, 2, 1], [48, 48]), ([2 ** 31 - 1, -2 ** 31], [2 ** 31 - 1])):
        y = P.shared_attention(s.q, cache, batch, P.SharedPrefix(_i32(first), _i32(prefix)))
        assert (y.float() - want).abs().max() <= 2.0 ** -7 * want.abs().max(), (first, prefix)
    # Offsets and lengths of rows: y is anything, and nothing else is touched.
    for cu, lens in (([0, 5, 2, 3], [60, 70, 80]), ([3, 1, 0, 0], [60, 70, 80]), ([-7, 1, 2, 900], [60, 70, 80]),
                     ([0, 1, 2, 3], [2 ** 31 - 1, -2 ** 31, 1 << 29]), ([2 ** 31 - 1, -1, 5, -2 ** 31], [1 << 30] * 3)):
        around = torch.full((5, 2, 64), 6.0, dtype=torch.bfloat16, device="cuda")
        odd = A.Batch(s.case.table.int(), _i32(lens), _i32(cu), rows=3)
        for first in ([0, 3], [1, 3], [0, 1]):
            P.shared_attention(s.q, cache, odd, P.SharedPrefix(_i32(first), _i32([48])), out=around[1:4])
            torch.cuda.synchronize()
            assert (around[0] == 6).all() and (around[4] == 6).all()
    none = P.SharedPrefix(_i32([0]), _i32([]))
    y = P.shared_attention(s.q, cache, batch, none)
    assert (y.float() - want).abs().max() <= 2.0 ** -7 * want.abs().max()
    empty = A.Batch(s.case.table.int()[:0], _i32([]))
    assert P.shared_attention(s.q[:0], cache, empty, none).shape == (0, 2, 64)


def test_rows_behind_the_batch_and_strided_tensors():
    log("padded")
    s = Step(128, 32, 2, 3, [(3, 64)], [9, 30, 4], [2, 1, 3], 9)
    rows = 10                                                 # 4 rows behind the last sequence
    wide = torch.full((rows, 6 * 128 + 40), 7.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((rows, 6 * 128 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:6, :768] = s.q.view(6, 768)
    batch = A.Batch(s.case.table.int(), _i32(s.lens), s.cu, rows=rows)
    q, y = wide[:, :768].view(rows, 6, 128), out[:, :768].view(rows, 6, 128)
    got = P.shared_attention(q, s.case.cache(), batch, s.shared(), out=y)
    assert got is y and (out[6:] == 3).all() and (out[:, 768:] == 3).all()
    T._compare(y[:6], None, s.case, s.q, s.counts, 128 ** -0.5, True, 0, T._some, False)


def test_runs_are_equal_on_any_stream_and_in_a_graph():
    log("captured")
    s = Step(128, 32, 2, 4, [(5, 1504), (3, 96)], [40, 9, 300, 2, 77, 5, 60, 1], [1] * 8, 3, False)
    cache, lens = s.case.cache(), _i32(s.lens)
    batch = A.Batch(s.case.table.int(), lens, max_len=max(s.lens))
    prefix = _i32([1504, 96])
    shared = P.SharedPrefix(_i32(s.first), prefix, max_len=1536, max_own=300)
    want = P.shared_attention(s.q, cache, batch, shared)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = P.shared_attention(s.q, cache, batch, shared, stream=side)
    ws = torch.empty(shared.workspace_bytes(cache, batch, 8), dtype=torch.uint8, device="cuda")
    q, y = s.q.clone(), torch.empty_like(s.q)
    with torch.cuda.stream(side):
        P.shared_attention(q, cache, batch, shared, out=y, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want) and torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.shared_attention(q, cache, batch, shared, out=y, workspace=ws)
    for i in range(4):                                        # shorter sequences and prefixes between eager calls
        q.copy_(s.q * (1 + i))
        lens.copy_(_i32([max(0, n - 13 * i) for n in s.lens]))
        prefix.copy_(_i32([1504 - 32 * i, 96 if i % 2 else 0]))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.shared_attention(q, cache, batch, shared)), i
        plain = A.attention(q, cache, batch).float()
        assert (y.float() - plain).abs().max() <= 2.0 ** -7 * plain.abs().max()
