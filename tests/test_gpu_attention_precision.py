"""GPU tests of the attention's probabilities far below the largest one, and of
values over pages of very different scales: the rows behind an attention sink.

Tolerances (before any run), against float64 on the same codes: a row's token j
has probability p_j = e_j / L with e_j = exp(s_j - the largest), L = sum e_j.
  - p_j enters the product with v in binary16: half a step, 2^-11 of it, or, below
    binary16's normal range, 2^-25 of what 1 stands for there.  The largest e_j is
    held as 2^9.5 at least, so 2^-34.5 in units of e_j;
  - values are held as code * 2^7 * their scale over the largest one, in binary16,
    whose smallest step is 2^-24: codes are multiples of 2^-9, so all are exact down to
    2^-22 of the largest scale; below, they are off by 2^-31 of it;
  - a score is off by (head_dim + 4) 2^-24 of the largest scale * sum |q_e k_e|,
    twice (numerator and denominator); exponentials 2^-20; sums (n / 16 + 32) 2^-24,
    twice; all of them on sum_j p_j |v_j|;
  - the result's rounding to bf16, 2^-8 of it.
Values have one sign and lie in few elements of a token (which ones goes by its
page), so that no element of y is small against its tolerance, and every page
weighs in some.  The comparison checks both: it has to refuse zeros, and, over
long sequences, the result with one page's values in another's place.
"""

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2609_04098_amd import attention as A
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
VALUES = torch.from_numpy(OA.E4M3_VALUES)


class Case:
    """One cache with its codes in natural order: k, v uint8 [pages, heads, page, dim]."""

    def __init__(self, dim, page, heads, lens, seed, k_scale=2.0 ** -6, v_scale=2.0 ** -3):
        self.gen = gen = torch.Generator("cuda").manual_seed(seed)
        self.dim, self.page, self.heads, self.lens = dim, page, heads, lens
        width = max(1, max(-(-n // page) for n in lens))
        n = len(lens) * width
        self.table = torch.randperm(n, generator=gen, device="cuda").view(len(lens), width)
        # Keys of both signs, codes of 2^-2 to 15; values of 1 to 1.9 in one element of 64, which one goes by the
        # page's place in its sequence, and 2^-6 of that in the others.
        sign = torch.randint(0, 2, (n, heads, page, dim), generator=gen, device="cuda", dtype=torch.uint8) * 128
        self.k = sign + torch.randint(0x28, 0x58, sign.shape, generator=gen, device="cuda", dtype=torch.uint8)
        self.v = torch.randint(0x08, 0x10, sign.shape, generator=gen, device="cuda", dtype=torch.uint8)
        place = torch.empty(n, dtype=torch.int64, device="cuda")
        place[self.table] = torch.arange(width, device="cuda").expand(len(lens), width)
        e = torch.arange(dim, device="cuda")
        self.v += 0x30 * ((e[None, :] * 5) % 64 == place[:, None] % 64)[:, None, None, :].to(torch.uint8)
        self.ks = torch.full((n, heads), k_scale, device="cuda")
        self.vs = torch.full((n, heads), v_scale, device="cuda")

    def at(self, b, t):
        """(page, slot) of a sequence's token."""
        return int(self.table[b, t // self.page]), t % self.page

    def cache(self):
        got = []
        for values, x in ((False, self.k), (True, self.v)):
            to = torch.empty(x.shape[0], x.shape[1], self.page * self.dim, dtype=torch.uint8, device="cuda")
            to[:, :, torch.from_numpy(OA.byte_places(self.page, self.dim, values)).cuda()] = x
            got.append(to)
        return A.KVCache(*got, self.ks, self.vs, self.page)

    def sequence(self, b, h, wrong=False):
        """(k, v, v's scales) of a sequence's tokens in float64; wrong: a page's values in another's place."""
        pages = self.table[b, :-(-self.lens[b] // self.page)]
        table = VALUES.cuda()
        of = lambda codes, scale, p: (table[codes[p, h].long()] * scale[p, h].double()[:, None, None]).reshape(-1, self.dim)
        of_values = pages.clone()
        if wrong:
            of_values[len(pages) // 2] = pages[len(pages) // 2 - 1]
        n = self.lens[b]
        return (of(self.k, self.ks, pages)[:n], of(self.v, self.vs, of_values)[:n],
                self.vs[pages, h].double().repeat_interleave(self.page)[:n])


def _compare(y, lse, case, q, counts, scale, causal, window, rows_of, pages):
    """Rows rows_of(n) of each sequence and the query heads of the first and last key heads."""
    group = q.shape[1] // case.heads
    row = 0
    for b, n in enumerate(counts):
        pick = sorted(set(rows_of(n)))
        for h in sorted({0, case.heads - 1}) if pick and case.lens[b] else []:
            k, v, vs = case.sequence(b, h)
            rows = torch.tensor([row + i for i in pick], device="cuda")
            own = slice(h * group, (h + 1) * group)
            x = q[rows, own].double().reshape(-1, case.dim)
            t = (case.lens[b] - n + torch.tensor(pick, device="cuda")).repeat_interleave(group)[:, None]
            j = torch.arange(case.lens[b], device="cuda")[None]
            seen = (j <= t) if causal else torch.ones(len(t), case.lens[b], dtype=torch.bool, device="cuda")
            if window:
                seen = seen & (j > t - window)
            s = (x @ k.T * scale).masked_fill(~seen, -np.inf)
            top = s.amax(1, keepdim=True)
            none = torch.isneginf(top[:, 0])
            e = torch.exp(s - torch.where(none[:, None], 0.0, top))
            total = e.sum(1, keepdim=True).clamp(min=1e-300)
            p = e / total
            want, size = p @ v, ((x.abs() @ k.abs().T) * abs(scale) * seen).amax(1, keepdim=True)
            score, sums = (case.dim + 4) * 2.0 ** -24 * size, (case.lens[b] / 16 + 32) * 2.0 ** -24
            held = torch.where(e > 0, torch.clamp(2.0 ** -11 * p, min=2.0 ** -34.5 / total), 0.0)
            off = torch.where(vs < 2.0 ** -22 * vs.max(), 2.0 ** -31 * vs.max(), 0.0)
            before = held @ v.abs() + (p @ v.abs()) * (2 * score + 2.0 ** -20 + 2 * sums) + (p @ off)[:, None]
            allowed = before + HALF * (want.abs() + before)
            got = y[rows, own].double().reshape(want.shape)
            bad = ~((got - want).abs() <= allowed)
            assert not bad.any(), (b, h, int(bad.sum()), bad.numel(), float(((got - want).abs() / want.abs()).nan_to_num().max()))
            assert not got[none].any()
            if (~none).any():      # a comparison that could fail
                live = want[~none]
                rms = live.square().mean().sqrt()
                assert (allowed[~none].square().mean().sqrt() < 0.05 * rms), float(allowed[~none].square().mean().sqrt() / rms)
                assert (live.abs() > allowed[~none]).all()
                if pages and case.lens[b] > 2 * case.page and not window:
                    other = (p @ case.sequence(b, h, wrong=True)[1])[-1]
                    assert ((other - want[-1]).abs() > allowed[-1]).any()
            if lse is not None:
                l = lse[rows, own].double().reshape(-1)
                assert torch.equal(torch.isneginf(l), none)
                ref = (top + total.log())[~none, 0]
                assert ((l[~none] - ref).abs() <= score[~none, 0] + 2.0 ** -20 + sums + 2.0 ** -22 * ref.abs()).all()
        row += n


def _some(n):
    return [i for i in (0, 1, n // 3, n // 2, n - 2, n - 1) if 0 <= i < n]


def _run(case, q, counts, scale=None, causal=True, window=0, max_len=None, rows_of=_some, pages=False):
    cu = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    lens = torch.tensor(case.lens, dtype=torch.int32, device="cuda")
    batch = A.Batch(case.table.int(), lens, cu, rows=sum(counts), max_len=max_len)
    scale = case.dim ** -0.5 if scale is None else scale
    y, lse = A.attention(q, case.cache(), batch, scale=scale, causal=causal, window=window, return_lse=True)
    _compare(y, lse, case, q, counts, scale, causal, window, rows_of, pages)


def _queries(case, rows, heads, scale=1.0):
    return (torch.randn(rows, heads, case.dim, generator=case.gen, device="cuda") * scale).to(torch.bfloat16)


SINKS = [      # dim, page, key heads, group, lengths, new rows (every kernel: test_gpu_attention_kernels.py)
    (128, 16, 1, 5, [300], [1]), (64, 32, 2, 4, [9000], [1]), (256, 32, 1, 4, [9000], [2]), (128, 64, 1, 8, [3000], [9]),
    (128, 32, 48, 4, [8200, 8200], [128, 128]), (256, 64, 32, 2, [4100], [260]), (64, 128, 2, 8, [8300], [5400]),
]


def add_sink(case, q_heads, counts, nats, at):
    """Queries, and keys changed so that a token at that share of each sequence's older ones, whose values become zero,
    scores so many nats where all others score about none (with a scale of 1)."""
    case.k[..., 0] = 0
    for b, n in enumerate(case.lens):
        if n == 0:
            continue
        p, slot = case.at(b, int((n - counts[b]) * at))
        case.k[p, :, slot] = 0
        case.k[p, :, slot, 0] = int(torch.tensor(16.0 * nats).to(torch.float8_e4m3fn).view(torch.uint8))
        case.v[p, :, slot] = 0
    case.ks.fill_(2.0 ** -4)
    q = _queries(case, sum(counts), q_heads, 1 / 64)
    q[..., 0] = 1.0
    return q


def _name(c):
    return "d%d_p%d_h%dx%d_%d" % (*c[:4], c[5][0])


@pytest.mark.parametrize("nats", [8, 14, 16, 18, 20])
@pytest.mark.parametrize("shape", SINKS, ids=_name)
def test_tokens_far_below_an_attention_sink(shape, nats):
    """One token whose values are zero, so many nats above all others: y is made of these."""
    dim, page, heads, group, lens, counts = shape
    log("sink %s %d nats" % (shape, nats))
    for at in (0, 0.7):
        case = Case(dim, page, heads, lens, seed=dim + page + nats)
        q = add_sink(case, heads * group, counts, nats, at)
        _run(case, q, counts, scale=1.0)


@pytest.mark.parametrize("shape", [SINKS[0], SINKS[2], SINKS[4], SINKS[5]], ids=_name)
def test_scores_that_grow(shape):
    """Scores that rise from token to token, by 52 nats in all, where the maximum has to follow all the way."""
    dim, page, heads, group, lens, counts = shape
    case = Case(dim, page, heads, lens, seed=dim)
    case.k[..., 0] = 0
    for b, n in enumerate(lens):
        t = torch.arange(n, device="cuda")                           # codes of 0 to 416 in order
        case.k[case.table[b, t // page], :, t % page, 0] = (t * 0x7E // n).to(torch.uint8)[:, None]
    case.ks.fill_(2.0 ** -3)
    q = _queries(case, sum(counts), heads * group, 1 / 64)
    q[..., 0] = 1.0
    _run(case, q, counts, scale=1.0)
    q[..., 0] = -1.0                                                 # and fall
    _run(case, q, counts, scale=1.0)


@pytest.mark.parametrize("apart", [10, 20, 22])
@pytest.mark.parametrize("shape", [SINKS[0], SINKS[1], SINKS[4], SINKS[5]], ids=_name)
def test_values_of_a_page_far_below_another(shape, apart):
    """The first page's values are 2^apart of the others', and nobody looks at them: the others stay exact."""
    dim, page, heads, group, lens, counts = shape
    case = Case(dim, page, heads, lens, seed=dim + apart)
    case.vs.fill_(2.0 ** -apart)
    for b in range(len(lens)):
        p = int(case.table[b, 0])
        case.vs[p] = 1.0
        case.k[p] = 0
        case.k[p, :, :, 0] = 0xFE                                    # -448
    case.ks.fill_(2.0 ** -2)
    q = _queries(case, sum(counts), heads * group, 1 / 256)
    q[..., 0] = 1.0
    _run(case, q, counts, scale=1.0)


@pytest.mark.parametrize("shape", [SINKS[0], SINKS[1], SINKS[3], SINKS[4]], ids=_name)
@pytest.mark.parametrize("exponent", [-118, -100, -60, 110])
def test_the_smallest_and_largest_value_scales(shape, exponent):
    """Results that are normal bf16 numbers, from scales at both ends of binary32's range."""
    dim, page, heads, group, lens, counts = shape
    case = Case(dim, page, heads, lens, seed=dim + exponent + 200, v_scale=2.0 ** exponent)
    _run(case, _queries(case, sum(counts), heads * group), counts)


@pytest.mark.parametrize("shape", [SINKS[0], SINKS[1], SINKS[3], SINKS[4]], ids=_name)
def test_scores_of_millions(shape):
    """The largest scores allowed: one token takes all, and y is its value exactly."""
    dim, page, heads, group, lens, counts = shape
    case = Case(dim, page, heads, lens, seed=dim + 1)
    case.k.zero_()
    best = {}
    for b, n in enumerate(lens):
        t = torch.randperm(n - counts[b], generator=case.gen, device="cuda")[:0x7E]
        case.k[case.table[b, t // page], :, t % page, 0] = torch.arange(len(t), device="cuda").to(torch.uint8)[:, None]
        best[b] = int(t[-1])
    case.ks.fill_(8.0)
    q = torch.zeros(sum(counts), heads * group, dim, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2048.0                                               # (up to 448 * 8 * 2048 = 7.3 million)
    cu = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    batch = A.Batch(case.table.int(), torch.tensor(lens, dtype=torch.int32, device="cuda"), cu, rows=sum(counts))
    y = A.attention(q, case.cache(), batch, scale=1.0)
    row = 0
    for b, n in enumerate(counts):
        p, slot = case.at(b, best[b])
        want = (VALUES.cuda()[case.v[p, :, slot].long()] * case.vs[p].double()[:, None]).repeat_interleave(group, 0)
        assert torch.equal(y[row:row + n].double(), want.expand(n, -1, -1))
        row += n


LONG = [      # dim, page, key heads, group, lengths, new rows, window, stated length
    (64, 128, 1, 2, [200000, 10], [2, 1], 0, 100), (256, 64, 1, 2, [100000], [3], 0, 100),
    (128, 64, 1, 8, [60000], [8187], 0, None), (64, 64, 1, 8, [16000], [8187], 0, None), (64, 64, 1, 8, [16000], [8187], 600, None),
    (256, 64, 8, 8, [2000, 1300, 50, 1999], [60, 40, 50, 50], 0, None), (128, 64, 2, 4, [131072, 77], [1, 1], 0, None),
    (128, 32, 2, 8, [40000, 5001, 3000, 3065], [7, 7, 1, 7], 3000, None), (64, 32, 2, 2, [40000, 20011], [1, 7], 0, None),
    (256, 16, 2, 3, [30000, 9000], [1, 1], 0, None),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", LONG, ids=lambda c: "d%d_h%dx%d_%d_w%d" % (c[0], c[2], c[3], c[4][0], c[6]))
def test_long_sequences(shape, causal):
    """Sequences over which random values would average away: every page's weight in y is seen."""
    dim, page, heads, group, lens, counts, window, stated = shape
    log("long %s causal %s" % (shape, causal))
    case = Case(dim, page, heads, lens, seed=dim + lens[0])
    _run(case, _queries(case, sum(counts), heads * group), counts, causal=causal, window=window, max_len=stated, pages=True)
