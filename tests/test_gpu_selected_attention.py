"""GPU tests of the pages' bounds, of the choice of pages and of the attention over them.

Bounds and choices are whole numbers and single roundings: everything is equal to the
oracle's.  The attention's tolerances: those of test_gpu_attention_precision.py, whose
cases these are."""

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import paging as OP
from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import paging as P
from tests import test_gpu_attention as G
from tests import test_gpu_attention_precision as T
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(counts):
    return [0] + list(np.cumsum(counts))


# ---------------------------------------------------------------- bounds

def _want_bounds(cache, table, lens, counts, codes, step):
    k = OA.E4M3_VALUES[G._oracle(cache).codes[0]]
    for b, n in enumerate(counts):
        length = min(max(lens[b], 0), table.shape[1] * cache.page_size)
        first = max(lens[b], 0) - n
        for entry in range(table.shape[1]):
            if n and (entry + 1) * cache.page_size <= length and (entry + 1) * cache.page_size > first \
                    and entry * cache.page_size < first + n:
                page = int(table[b, entry])
                if 0 <= page < k.shape[0]:
                    for h in range(cache.kv_heads):
                        codes[page, h], step[page, h] = OP.page_bounds(k[page, h], float(cache.k_scale[page, h]))
    return codes, step


@pytest.mark.parametrize("dim,page,heads,lens,counts", [
    (64, 16, 1, [16], None), (128, 32, 3, [64, 63, 65, 32, 1], None), (256, 64, 2, [128, 64], None),
    (64, 128, 5, [128, 300, 256], [1, 100, 256]), (128, 16, 2, [50, 0, 33, 16, 7], [50, 0, 17, 2, 7]),
    (256, 16, 4, [100, 48], [70, 33]), (128, 128, 1, [640], [520]), (64, 16, 8, [17 * i for i in range(80)], [i % 40 for i in range(80)]),
    (128, 32, 2, [5, 40, 1 << 30], [9, 200, 70])])
def test_page_bounds(dim, page, heads, lens, counts):
    log("bounds %s" % ((dim, page, heads, lens[:4]),))
    gen = torch.Generator().manual_seed(dim + page + sum(lens) % 1000)
    width = max(1, max(-(-min(n, 700 if n < 1 << 20 else 96) // page) for n in lens))
    n_pages = len(lens) * width + 2
    table = torch.randperm(n_pages, generator=gen)[:len(lens) * width].view(len(lens), width).int()
    cache = G._random_cache(gen, n_pages, heads, page, dim, nan=False)
    cache.k[0] &= 0x80                                            # zeros of both signs
    cache.k_scale[1] *= 0.7
    bounds = P.PageBounds(torch.full((n_pages, heads, 2, dim), -77, dtype=torch.int8, device="cuda"),
                          torch.full((n_pages, heads), -7.0, device="cuda"))
    want = _want_bounds(cache, table, lens, counts or [1] * len(lens), bounds.codes.cpu().numpy().astype(np.int64),
                        bounds.step.cpu().numpy())
    batch = A.Batch(table.cuda(), _i32(lens), None if counts is None else _i32(_cu(counts)),
                    rows=None if counts is None else sum(counts) + 3)
    P.page_bounds(cache, batch, bounds)
    assert np.array_equal(bounds.codes.cpu().numpy(), want[0]) and np.array_equal(bounds.step.cpu().numpy(), want[1])


def test_bounds_of_pages_outside_the_cache_and_strided_buffers():
    gen = torch.Generator().manual_seed(3)
    cache = G._random_cache(gen, 6, 2, 16, 64, nan=False)
    pool = torch.zeros(6, 3, 2, 2, 64, dtype=torch.int8, device="cuda")
    steps = torch.zeros(6, 5, device="cuda")
    bounds = P.PageBounds(pool[:, 1], steps[:, 1:3])
    table = torch.tensor([[0, 9], [-1, 2], [5, 1 << 30]], dtype=torch.int32)
    lens, counts = [32, 32, 40], [32, 20, 40]
    P.page_bounds(cache, A.Batch(table.cuda(), _i32(lens), _i32(_cu(counts)), rows=sum(counts)), bounds)
    want = _want_bounds(cache, table, lens, counts, np.zeros((6, 2, 2, 64), dtype=np.int64), np.zeros((6, 2), dtype=np.float32))
    assert np.array_equal(bounds.codes.cpu().numpy(), want[0]) and np.array_equal(bounds.step.cpu().numpy(), want[1])
    assert not pool[:, [0, 2]].any() and not steps[:, [0, 3, 4]].any()


# ---------------------------------------------------------------- choice

def _want_choice(q, cache, bounds, table, lens, counts, count, first, recent, causal):
    """Per row (None: behind the last sequence): (token, key heads' lists)."""
    q, group = q.double().cpu().numpy(), q.shape[1] // cache.kv_heads
    codes, step = bounds.codes.cpu().numpy().astype(np.int64), bounds.step.cpu().numpy()
    got, most = [], table.shape[1] * cache.page_size
    for b, n in enumerate(counts):
        for i in range(n):
            length = min(max(lens[b], 0), most)
            t = min(max(lens[b], 0) - n + i, length - 1) if causal else length - 1
            seen = 0 if t < 0 else t // cache.page_size + 1
            heads = []
            for h in range(cache.kv_heads):
                qi, units = OP.query_codes(q[len(got), h * group:(h + 1) * group])
                scores = [None] * seen
                for j in range(first, seen - recent if seen > count else 0):
                    page = int(table[b, j])
                    if 0 <= page < codes.shape[0]:
                        scores[j] = OP.page_score(qi, units, codes[page, h], step[page, h])
                heads.append(OP.choose(scores, seen, count, first, recent))
            got.append((t, heads))
    return got


def _check_choice(sel, want, cache, table, counts, count):
    index, pages, tokens = sel.index.cpu(), sel.pages.cpu(), sel.tokens.tolist()
    seq = [b for b, n in enumerate(counts) for _ in range(n)]
    for r, (t, heads) in enumerate(want):
        for h, some in enumerate(heads):
            assert index[r, h].tolist() == some + [-1] * (count - len(some)), (r, h)
            assert pages[r, h].tolist() == [int(table[seq[r], j]) for j in some] + [-1] * (count - len(some))
        n = len(heads[0])
        assert tokens[r] == (0 if n == 0 else (n - 1) * cache.page_size + t % cache.page_size + 1)
    assert tokens[len(want):] == [-1] * (len(tokens) - len(want))


def _all_bounds(cache):
    """Bounds of every page, by the oracle."""
    k = OA.E4M3_VALUES[G._oracle(cache).codes[0]]
    n, h = k.shape[:2]
    codes, step = np.zeros((n, h, 2, cache.head_dim), dtype=np.int8), np.zeros((n, h), dtype=np.float32)
    for p in range(n):
        for i in range(h):
            codes[p, i], step[p, i] = OP.page_bounds(k[p, i], float(cache.k_scale[p, i]))
    return P.PageBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(step).cuda())


CHOICES = [      # dim, page, key heads, group, lengths, new rows (None: one each), count, first, recent, causal
    (64, 16, 1, 1, [400], None, 6, 1, 1, True), (128, 16, 2, 5, [300, 17, 0, 90, 1], None, 5, 1, 2, True),
    (256, 16, 1, 3, [500, 333], None, 9, 0, 1, True), (128, 32, 3, 8, [640, 100, 64], [3, 0, 5], 4, 2, 1, True),
    (64, 16, 2, 16, [700, 16], [6, 16], 7, 0, 3, True), (64, 16, 1, 17, [300], [2], 4, 1, 1, True),
    (128, 16, 1, 40, [200, 250], None, 3, 1, 1, True), (64, 64, 2, 4, [900, 800], [4, 3], 3, 1, 1, False),
    (128, 16, 2, 2, [130, 90], [4, 100], 8, 3, 5, True), (64, 16, 1, 2, [16 * 700 + 3], None, 300, 1, 2, True),
    (64, 16, 1, 4, [16 * 600, 16 * 513 + 1], None, 511, 0, 1, True), (128, 16, 1, 4, [100, 60], None, 1, 0, 1, True)]


@pytest.mark.parametrize("c", CHOICES, ids=lambda c: "_".join(str(x) for x in c[:4]) + "_%d_of_%d" % (c[6], c[4][0]))
def test_select_pages(c):
    dim, page, heads, group, lens, counts, count, first, recent, causal = c
    log("select %s" % (c,))
    gen = torch.Generator().manual_seed(dim + sum(lens))
    counts = counts or [1] * len(lens)
    width = max(-(-n // page) for n in lens)
    n_pages = len(lens) * width + 1
    table = torch.randperm(n_pages, generator=gen)[:len(lens) * width].view(len(lens), width).int()
    cache = G._random_cache(gen, n_pages, heads, page, dim, nan=False)
    bounds = _all_bounds(cache)
    rows = sum(counts) + (2 if c[5] else 0)
    q = G._bf16(gen, rows, heads * group, dim).cuda()
    batch = A.Batch(table.cuda(), _i32(lens), _i32(_cu(counts)) if c[5] else None, rows=rows)
    out = P.Selection(*[torch.full((rows, heads, count), -9, dtype=torch.int32, device="cuda") for _ in range(2)], _i32([9] * rows))
    sel = P.select_pages(q, cache, batch, bounds, count, first, recent, causal, out=out)
    assert sel is out
    _check_choice(sel, _want_choice(q, cache, bounds, table, lens, counts, count, first, recent, causal), cache, table, counts,
                  count)
    assert (sel.index[sum(counts):] == -9).all() and (sel.pages[sum(counts):] == -9).all()


def test_ties_zeros_and_pages_outside_the_cache():
    """Equal scores go to the lowest pages, over more than a round of the selection's
    threads; pages that are not there come last."""
    log("ties")
    gen = torch.Generator().manual_seed(1)
    width, n_pages = 1300, 7
    cache = G._random_cache(gen, n_pages, 2, 16, 64, nan=False)
    bounds = _all_bounds(cache)
    for low, high in ((0, 3), (0, 1), (-2, 9)):
        table = torch.randint(low, high, (3, width), generator=gen, dtype=torch.int32)
        q = G._bf16(gen, 3, 4, 64).cuda()
        q[1] = 0
        lens = [width * 16, width * 16 - 3, 16 * 600]
        batch = A.Batch(table.cuda(), _i32(lens))
        for count in (2, 100, 513, 1299):
            sel = P.select_pages(q, cache, batch, bounds, count, first=1 if count > 2 else 0)
            want = _want_choice(q, cache, bounds, table, lens, [1] * 3, count, 1 if count > 2 else 0, 1, True)
            _check_choice(sel, want, cache, table, [1] * 3, count)


def test_more_pages_than_lds_holds():
    """Tables of over 8192 pages: keys in memory, several runs of the selection's rounds."""
    log("many pages")
    gen = torch.Generator().manual_seed(9)
    n_pages, width = 300, 20000
    cache = G._random_cache(gen, n_pages, 1, 16, 64, nan=False)
    bounds = _all_bounds(cache)
    table = torch.randint(0, n_pages, (2, width), generator=gen, dtype=torch.int32)
    q = G._bf16(gen, 2, 3, 64).cuda()
    lens = [width * 16 - 5, 16 * 8200]
    batch = A.Batch(table.cuda(), _i32(lens))
    # (each page stands in a table many times: its score is looked up)
    codes, step = bounds.codes.cpu().numpy().astype(np.int64), bounds.step.cpu().numpy()
    for count in (3, 2000, 8190, 19000):
        sel = P.select_pages(q, cache, batch, bounds, count)
        want = []
        for r, n in enumerate(lens):
            qi, units = OP.query_codes(q[r].double().cpu().numpy())
            of = [OP.page_score(qi, units, codes[p, 0], step[p, 0]) for p in range(n_pages)]
            seen = (n - 1) // 16 + 1
            want.append((n - 1, [OP.choose([of[p] for p in table[r].tolist()], seen, count, 1, 1)]))
        _check_choice(sel, want, cache, table, [1, 1], count)


def test_lengths_that_make_no_sense():
    log("lengths")
    gen = torch.Generator().manual_seed(2)
    cache = G._random_cache(gen, 30, 1, 16, 64, nan=False)
    bounds = _all_bounds(cache)
    table = torch.randint(0, 30, (5, 8), generator=gen, dtype=torch.int32)
    q = G._bf16(gen, 9, 2, 64).cuda()
    lens, counts = [-5, 2 ** 31 - 1, 1 << 29, 128, 3], [1, 2, 1, 1, 4]
    batch = A.Batch(table.cuda(), _i32(lens), _i32(_cu(counts)), rows=9)
    for causal in (True, False):
        sel = P.select_pages(q, cache, batch, bounds, 4, causal=causal)
        _check_choice(sel, _want_choice(q, cache, bounds, table, lens, counts, 4, 1, 1, causal), cache, table, counts, 4)
        y = P.selected_attention(q, cache, sel)
        assert torch.isfinite(y.float()).all() and not y[0].any()
    none = A.Batch(torch.zeros(2, 0, dtype=torch.int32, device="cuda"), _i32([0, 7]))
    sel = P.select_pages(q[:2], cache, none, bounds, 4)
    assert sel.tokens.tolist() == [0, 0] and (sel.index == -1).all()
    assert not P.selected_attention(q[:2], cache, sel).any()
    empty = A.Batch(table[:0].cuda(), _i32([]))
    sel = P.select_pages(q[:0], cache, empty, bounds, 4)
    assert P.selected_attention(q[:0], cache, sel).shape == (0, 2, 64)


# ---------------------------------------------------------------- attention

def _compare(y, lse, case, q, sel, scale, rows):
    """As test_gpu_attention_precision._compare, over the selection's tokens."""
    group = q.shape[1] // case.heads
    table = T.VALUES.cuda()
    for r in rows:
        n = int(sel.tokens[r])
        for h in sorted({0, case.heads - 1}):
            own = slice(h * group, (h + 1) * group)
            got = y[r, own].double()
            if n <= 0:
                assert not got.any() and (lse is None or torch.isneginf(lse[r, own]).all())
                continue
            pages = sel.pages[r, h, :-(-n // case.page)].long()
            of = lambda codes, s: (table[codes[pages, h].long()] * s[pages, h].double()[:, None, None]).reshape(-1, case.dim)[:n]
            k, v = of(case.k, case.ks), of(case.v, case.vs)
            vs = case.vs[pages, h].double().repeat_interleave(case.page)[:n]
            x = q[r, own].double()
            s = x @ k.T * scale
            top = s.amax(1, keepdim=True)
            e = torch.exp(s - top)
            total = e.sum(1, keepdim=True)
            p = e / total
            want, size = p @ v, ((x.abs() @ k.abs().T) * abs(scale)).amax(1, keepdim=True)
            score, sums = (case.dim + 4) * 2.0 ** -24 * size, (n / 16 + 32) * 2.0 ** -24
            held = torch.clamp(2.0 ** -11 * p, min=2.0 ** -34.5 / total)
            off = torch.where(vs < 2.0 ** -22 * vs.max(), 2.0 ** -31 * vs.max(), 0.0)
            before = held @ v.abs() + (p @ v.abs()) * (2 * score + 2.0 ** -20 + 2 * sums) + (p @ off)[:, None]
            bad = ~((got - want).abs() <= before + HALF * (want.abs() + before))
            assert not bad.any(), (r, h, int(bad.sum()), float((got - want).abs().max()))
            if lse is not None:
                ref = (top + total.log())[:, 0]
                assert ((lse[r, own].double() - ref).abs() <= score[:, 0] + 2.0 ** -20 + sums + 2.0 ** -22 * ref.abs()).all()


@pytest.mark.parametrize("dim,page,heads,group,lens,counts,count", [
    (64, 16, 1, 1, [400], None, 6), (128, 16, 8, 5, [900, 17, 0, 90, 1], None, 24), (256, 16, 1, 3, [500, 333], None, 9),
    (128, 64, 2, 8, [9000], None, 64), (64, 128, 2, 4, [6000, 5000], [4, 3], 20), (256, 32, 2, 8, [5000, 3000], [3, 2], 40),
    (128, 16, 1, 40, [2000, 250], None, 30), (64, 16, 2, 32, [700], [9], 20), (256, 32, 1, 20, [700, 30], None, 12),
    (128, 32, 4, 4, [700] * 40, None, 9), (64, 16, 1, 130, [3000] * 3, None, 60), (128, 16, 1, 128, [900] * 40, [2] * 40, 30),
    (256, 16, 1, 100, [600] * 20, None, 20), (64, 64, 8, 8, [4000] * 30, None, 30), (128, 16, 3, 7, [1000, 33], [2, 5], 500)])
def test_selected_attention(dim, page, heads, group, lens, counts, count):
    log("selected %s" % ((dim, page, heads, group, lens[:3], count),))
    case = T.Case(dim, page, heads, lens, dim + lens[0])
    rows = sum(counts) if counts else len(lens)
    q = T._queries(case, rows, heads * group)
    cache = case.cache()
    bounds = P.alloc_page_bounds(cache)
    P.page_bounds(cache, A.Batch(case.table.int(), _i32(lens), _i32(_cu(lens)), rows=sum(lens)), bounds)
    batch = A.Batch(case.table.int(), _i32(lens), _i32(_cu(counts)) if counts else None, rows=rows)
    sel = P.select_pages(q, cache, batch, bounds, count)
    some = sorted({0, 1, rows // 2, rows - 1} & set(range(rows)))
    for scale in (dim ** -0.5, -0.03):
        y, lse = P.selected_attention(q, cache, sel, scale=scale, return_lse=True)
        _compare(y, lse, case, q, sel, scale, some)
    again = P.selected_attention(q, cache, sel, scale=-0.03)
    assert torch.equal(y, again)
    if count * page >= max(lens):                                 # all pages taken: the attention itself
        plain = A.attention(q, cache, batch).float()
        full = P.selected_attention(q, cache, sel).float()
        assert (plain - full).abs().max() <= 2.0 ** -7 * plain.abs().max()
    sel.tokens[0] = -1                                            # a row that is left as it is
    out = torch.full_like(q, 5.0)
    P.selected_attention(q, cache, sel, out=out)
    assert (out[0] == 5).all() and torch.equal(out[1:], P.selected_attention(q, cache, sel)[1:])


def test_a_choice_of_the_callers_own():
    """Pages in any order, the same one twice, pages that are not there (masked), NaN
    behind the tokens."""
    log("own choice")
    case = T.Case(128, 16, 2, [800], 7)
    case.k[:, :, 9:], case.v[:, :, 9:] = 0x7F, 0xFF
    q = T._queries(case, 2, 8)
    pages = _i32([[[5, 3, 3, 40], [1, 0, 7, 2]], [[9, 9, 9, 9], [30, 31, 3, 1]]])
    sel = P.Selection(torch.zeros_like(pages), pages, _i32([9, 9]))
    _compare(*P.selected_attention(q, case.cache(), sel, return_lse=True), case, q, sel, 128 ** -0.5, [0, 1])
    case = T.Case(128, 16, 2, [800], 8)
    sel = P.Selection(torch.zeros_like(pages), pages, _i32([64, 1 << 30]))      # cut to what there is
    y, lse = P.selected_attention(q, case.cache(), sel, return_lse=True)
    sel.tokens[1] = 64
    _compare(y, lse, case, q, sel, 128 ** -0.5, [0, 1])
    gone = pages.clone()
    gone[0, :, 1], gone[1, :, 2] = -3, 1 << 30
    with_less = torch.cat((pages[:, :, :1], pages[:, :, 2:], pages[:, :, :1]), dim=2)
    with_less[1] = torch.cat((pages[1, :, :2], pages[1, :, 3:], pages[1, :, :1]), dim=1)
    y = P.selected_attention(q, case.cache(), P.Selection(gone, gone, _i32([64, 64])))
    less = P.Selection(with_less.contiguous(), with_less.contiguous(), _i32([48, 48]))
    _compare(y, None, case, q, less, 128 ** -0.5, [0, 1])


def test_far_pages():
    """Pages whose bytes and bounds lie beyond 2^32, by strides."""
    log("far pages")
    n, stride = 70, 1 << 26
    pool = torch.zeros(n * stride, dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    dim, page = 64, 16
    case = T.Case(dim, page, 1, [page * n], 3)
    near = case.cache()
    far = [torch.as_strided(pool, (n, 1, page * dim), (stride, page * dim, 1), at) for at in (0, 4096)]
    for to, x in zip(far, (near.k, near.v)):
        to.copy_(x)
    codes = torch.as_strided(pool.view(torch.int8), (n, 1, 2, dim), (stride, 2 * dim, dim, 1), 8192)
    cache = A.KVCache(*far, near.k_scale, near.v_scale, page)
    bounds = P.PageBounds(codes, torch.zeros(n, 1, device="cuda"))
    whole = A.Batch(case.table.int(), _i32([page * n]), _i32([0, page * n]), rows=page * n)
    P.page_bounds(cache, whole, bounds)
    plain = P.alloc_page_bounds(near)
    P.page_bounds(near, whole, plain)
    assert torch.equal(bounds.codes, plain.codes) and torch.equal(bounds.step, plain.step)
    q = T._queries(case, 1, 4)
    batch = A.Batch(case.table.int(), _i32([page * n]))
    a, b = P.select_pages(q, cache, batch, bounds, 9), P.select_pages(q, near, batch, plain, 9)
    assert torch.equal(a.index, b.index)
    assert torch.equal(P.selected_attention(q, cache, a), P.selected_attention(q, near, b))


# ---------------------------------------------------------------- together

def _serve(steps, captured):
    """Steps of a loop: tables, append, bounds, choice, attention, one layer; requests that
    come, draft, are rejected and end.  Checked against the oracle's cache and choice."""
    gen = torch.Generator().manual_seed(steps)
    dim, page, heads, group, n, width, rows = 64, 16, 2, 3, 4, 24, 64
    r = P.alloc_requests(n, width, 60, page, "cuda")
    cache = A.alloc_kv_cache(60, heads, dim, page, "cuda")
    cache.k.zero_(), cache.v.zero_()
    bounds = P.alloc_page_bounds(cache)
    rope = A.Rope(G._inv_freq(32).cuda())
    step = P.Step(r, rows)
    new, drop = _i32([0] * n), _i32([0] * n)
    x = torch.zeros(rows, (group + 2) * heads * dim, dtype=torch.bfloat16, device="cuda")
    q, k, v = (x[:, a * heads * dim:b * heads * dim].view(rows, -1, dim) for a, b in
               ((0, group), (group, group + 1), (group + 1, group + 2)))
    sel = P.Selection(*[torch.zeros(rows, heads, 5, dtype=torch.int32, device="cuda") for _ in range(2)], _i32([0] * rows))
    y = torch.zeros(rows, heads * group, dim, dtype=torch.bfloat16, device="cuda")

    def run():
        P.step_tables(r, new, rows, drop, out=step)
        A.kv_append(cache, step.batch, k, v, rope=rope)
        P.page_bounds(cache, step.batch, bounds)
        P.select_pages(q, cache, step.batch, bounds, 5, out=sel)
        P.selected_attention(q, cache, sel, out=y)

    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
    want = OP.Pool(r.page_table.cpu().tolist(), r.kv_len.tolist(), r.free_pages.tolist(), 60, page)
    oracle = G._oracle(cache)
    plans = [([50, 3, 0, 9], [0] * 4), ([1, 1, 60, 1], [0] * 4), ([5, 5, 5, 5], [0] * 4), ([4, 4, 1, 1], [3, 5, 2, 0]),
             ([30, 0, 1, 1], [10 ** 9, 0, 0, 0]), ([16, 16, 16, 16], [0, 1, 0, 0]), ([1, 1, 1, 1], [0, 0, 10 ** 9, 0])]
    for i in range(steps):
        a, d = plans[i % len(plans)]
        x.copy_(G._bf16(gen, *x.shape))
        new.copy_(_i32(a)), drop.copy_(_i32(d))
        y.fill_(3.0)
        graph.replay() if captured else run()
        torch.cuda.synchronize()
        cu, pos, slots = want.step(a, d, [0] * 4, rows)
        counts = list(np.diff(cu))
        assert step.batch.cu_rows.tolist() == list(cu) and r.page_table.tolist() == want.table
        table = r.page_table.cpu().numpy()
        kr = OA.norm_rope(G._np(k)[:cu[-1]], None, 0.0, pos, G._inv_freq(32).numpy(), False)
        starts = [want.kv_len[b] - counts[b] for b in range(n)]
        oracle.append(table, starts, counts, kr, G._np(v)[:cu[-1]])
        G._same_cache(cache, oracle, "step %d" % i)
        ref = _want_choice(q, cache, bounds, table, want.kv_len, counts, 5, 1, 1, True)
        _check_choice(sel, ref, cache, table, counts, 5)
        # Every full page has its bounds.
        held = P.PageBounds(torch.zeros_like(bounds.codes), torch.zeros_like(bounds.step))
        full = [(b, e) for b in range(n) for e in range(want.kv_len[b] // page)]
        c, s = _want_bounds(cache, table, want.kv_len, want.kv_len, held.codes.cpu().numpy().astype(np.int64), held.step.cpu().numpy())
        at = [int(table[b, e]) for b, e in full]
        assert np.array_equal(bounds.codes.cpu().numpy()[at], c[at]) and np.array_equal(bounds.step.cpu().numpy()[at], s[at])
        # Rows over the chosen pages, as a sequence of their own.
        for row in sorted({0, int(cu[-1]) // 2, int(cu[-1]) - 1}):
            for h in range(heads):
                got_n = int(sel.tokens[row])
                some = sel.pages[row, h].cpu().numpy()[None]
                w, _, size, absolute, most = OA.attention(G._np(q)[row:row + 1], oracle, some, [got_n], [1], dim ** -0.5, False, 0)
                own = slice(h * group, (h + 1) * group)
                before = absolute[0, own] * (2.0 ** -11 + 2 * (dim + 4) * 2.0 ** -24 * size[0, own, None] + 2.0 ** -20) \
                    + 2.0 ** -25 * most[0, own, None]
                assert (np.abs(G._np(y)[row, own] - w[0, own]) <= before + HALF * (np.abs(w[0, own]) + before)).all()
        assert (y[int(cu[-1]):] == 3).all()


@pytest.mark.parametrize("captured", [False, True])
def test_a_serving_loop(captured):
    log("serving loop, captured %s" % captured)
    _serve(9, captured)
