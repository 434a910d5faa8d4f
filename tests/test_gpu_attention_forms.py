"""GPU tests of the forms that the attention takes by the sizes of a step: tiles
of 128 rows, whole and in pieces, many sequences, heads over more than one tile,
scales that are no powers of two, pages that sequences share, captured steps.

Sampled rows of every sequence are compared with float64.  Tolerances: those of
test_gpu_attention.py, with the sums' part written out: a row's sum of
exponentials and its products are added in chains of at most one link for 16
tokens, each rounded to binary32, and 32 links more in joins and within a tile,
so (n / 16 + 32) 2^-24 of the sum.
"""

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2609_04098_amd import attention as A
from tests.gpu_common import log
from tests.test_gpu_attention import HALF, _cu, _i32, _same_cache

pytestmark = pytest.mark.gpu


def _codes(gen, pages, heads, page, dim):
    """Random codes, no NaN."""
    c = torch.randint(0, 254, (pages, heads, page * dim), generator=gen, device="cuda", dtype=torch.int32)
    return (c + (c >= 127)).to(torch.uint8)


def _cache(gen, pages, heads, page, dim, powers=True):
    scales = []
    for _ in range(2):
        s = torch.exp2(torch.randint(-12, -6, (pages, heads), generator=gen, device="cuda").float())
        scales.append(s if powers else s * (1 + torch.rand(pages, heads, generator=gen, device="cuda")))
    return A.KVCache(_codes(gen, pages, heads, page, dim), _codes(gen, pages, heads, page, dim), *scales, page)


def _spoil(cache, table, lens):
    """NaN codes behind each sequence's last token, in the page that it ends in."""
    p, d = cache.page_size, cache.head_dim
    k = cache.k.view(-1, cache.kv_heads, p // 16, d // 16, 16, 16)
    v = cache.v.view(-1, cache.kv_heads, p // 16, d // 64, 4, 16, 4, 4)
    for b, n in enumerate(lens):
        for t in range(n, -(-n // p) * p):
            page, g, u = int(table[b, t // p]), t % p // 16, t % 16
            k[page, :, g, :, u] = 0x7F
            v[page, :, g, :, u // 4, :, :, u % 4] = 0xFF


def _compare(y, lse, cache, q, table, lens, counts, scale, causal, window, heads, rows_of):
    """Rows rows_of(n) of each sequence and all query heads of the key heads `heads`."""
    group = q.shape[1] // cache.kv_heads
    row = 0
    for b, n in enumerate(counts):
        pick = sorted(set(rows_of(n)))
        for h in heads if pick and lens[b] else []:
            pages = table[b, :-(-lens[b] // cache.page_size)].long()
            there = pages < cache.k.shape[0]
            at = torch.where(there, pages, 0).cuda()
            one = OA.Cache.from_bytes(cache.k[at, h:h + 1].cpu().numpy(), cache.v[at, h:h + 1].cpu().numpy(),
                                      cache.k_scale[at, h:h + 1].cpu().double().numpy(),
                                      cache.v_scale[at, h:h + 1].cpu().double().numpy(), cache.page_size)
            order = np.arange(len(pages))
            k, _ = one.sequence(0, order, 0, lens[b])
            v, _ = one.sequence(1, order, 0, lens[b])
            of_token = np.arange(lens[b]) // cache.page_size
            there = there.numpy()[of_token]
            k, v = np.where(there[:, None], k, 0.0), np.where(there[:, None], v, 0.0)
            rows = torch.tensor([row + i for i in pick], device=q.device)
            own = slice(h * group, (h + 1) * group)
            x = q[rows, own].double().cpu().numpy().reshape(-1, cache.head_dim)
            t = np.repeat(lens[b] - n + np.array(pick), group)[:, None]
            j = np.arange(lens[b])[None]
            seen = there[None] & ((j <= t) if causal else True) & ((j > t - window) if window else True)
            s = np.where(seen, (x @ k.T) * scale, -np.inf)
            m = s.max(1, keepdims=True)
            w = np.where(seen, np.exp(s - np.where(np.isneginf(m), 0.0, m)), 0.0)
            total = w.sum(1, keepdims=True)
            none = total[:, 0] == 0
            total[none] = 1.0
            size = np.where(seen, (np.abs(x) @ np.abs(k).T) * abs(scale), 0.0).max(1, keepdims=True)
            sums = (lens[b] / 16 + 32) * 2.0 ** -24
            score = (cache.head_dim + 4) * 2.0 ** -24 * size
            want = (w / total) @ v
            most = seen.sum(1, keepdims=True) * 448.0 * float(one.scale[1].max())
            before = ((w / total) @ np.abs(v)) * (2.0 ** -11 + 2 * score + 2.0 ** -20 + 2 * sums) + 2.0 ** -25 * most
            got = y[rows, own].double().cpu().numpy().reshape(want.shape)
            bad = ~(np.abs(got - want) <= before + HALF * (np.abs(want) + before))
            assert not bad.any(), (b, h, bad.sum(), bad.size, float(np.nanmax(np.abs(got - want))))
            assert not got[none].any()
            if lse is not None:
                l = lse[rows, own].double().cpu().numpy().reshape(-1)
                assert np.array_equal(np.isneginf(l), none)
                ref = m[~none, 0] + np.log(total[~none, 0])
                assert np.all(np.abs(l[~none] - ref) <= score[~none, 0] + 2.0 ** -20 + sums + 2.0 ** -22 * np.abs(ref))
        row += n


def _run(dim, page, hkv, group, lens, counts, causal=True, window=0, powers=True, cut=(), max_len=None, seed=0,
         heads=None, every=None, shared=False, cu=True):
    log("attention forms %s" % ((dim, page, hkv, group, len(lens), sum(counts), causal, window, powers),))
    gen = torch.Generator("cuda").manual_seed(seed + dim + page)
    width = max(1, max(-(-n // page) for n in lens))
    pages = len(lens) * width
    table = torch.randperm(pages, generator=gen, device="cuda").view(len(lens), width).cpu()
    if shared:
        table[:, 0] = table[0, 0]
    cache = _cache(gen, pages, hkv, page, dim, powers)
    if not shared:
        _spoil(cache, table, lens)
    for b, x in cut:
        table[b, x] = 2 ** 31 - 1
    behind = 5 if cu else 0
    rows = sum(counts)
    q = torch.randn(rows + behind, hkv * group, dim, generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)) if cu else None, rows=rows + behind, max_len=max_len)
    y, lse = A.attention(q, cache, batch, causal=causal, window=window, out=out, return_lse=True)
    assert (out[rows:] == 7.0).all()
    ends = every or (lambda n: [i for i in (0, 1, n // 3, n // 2, n - 2, n - 1) if 0 <= i < n])
    _compare(y, lse, cache, q, table, lens, counts, dim ** -0.5, causal, window, heads or sorted({0, hkv // 2, hkv - 1}), ends)
    return batch.workspace_bytes(cache, hkv * group)


TILES = [      # dim, page, key heads, group, lengths, new rows
    (128, 16, 32, 8, [300, 70, 700, 257], [64, 70, 65, 57]),
    (128, 64, 48, 5, [40, 0, 600, 333], [40, 0, 200, 120]),
    (64, 128, 32, 4, [130, 400, 1000, 97], [130, 100, 99, 97]),
    (256, 32, 32, 2, [300, 240], [75, 60]),
    (256, 16, 33, 3, [100, 33, 400], [90, 33, 40]),
]


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 50), (False, 130), (True, 1)])
@pytest.mark.parametrize("case", TILES, ids=lambda c: "d%d_p%d_h%dx%d" % c[:4])
def test_tiles_of_128_rows(case, causal, window):
    dim, _, hkv, group, lens, counts = case
    each = -(-sum(counts) * group // len(lens))
    assert each > 64 and -(-each // 128) * len(lens) * hkv >= (128 if dim == 256 else 512)
    _run(*case, causal, window, seed=window)


@pytest.mark.parametrize("case", [TILES[0], TILES[2], TILES[4], (128, 32, 2, 4, [500, 90], [1, 70]),
                                  (256, 64, 1, 6, [300], [2])], ids=lambda c: "d%d_p%d_h%dx%d" % c[:4])
def test_scales_that_are_no_powers_of_two(case):
    _run(*case, powers=False, seed=3)
    _run(*case, powers=False, window=70, seed=4)


@pytest.mark.parametrize("dim,hkv,group,lens,counts", [
    (256, 8, 8, [2000, 1300, 50, 1999], [60, 40, 50, 50]), (256, 32, 2, [1500, 700], [65, 65]),
    (128, 1, 8, [60000], [8187]), (64, 1, 8, [16000], [8187])])
def test_tiles_of_128_rows_in_pieces(dim, hkv, group, lens, counts):
    assert _run(dim, 64, hkv, group, lens, counts, seed=5, heads=[0, hkv - 1]) > 0
    _run(dim, 64, hkv, group, lens, counts, seed=6, heads=[hkv // 2], window=600)
    _run(dim, 64, hkv, group, lens, counts, seed=7, heads=[hkv // 2], causal=False, powers=False)


@pytest.mark.parametrize("dim,group,window", [(128, 8, 3000), (64, 2, 1025), (256, 3, 4096), (128, 40, 700), (128, 5, 1)])
@pytest.mark.parametrize("new", [1, 7])
def test_windows_of_long_sequences_in_pieces(dim, group, window, new):
    """Pieces begin where a tile's window does; its tokens next to the borders."""
    assert _run(dim, 32, 2, group, [40000, 5001, window, window + 65], [new, new, 1, new], window=window, seed=8, every=range) > 0
    _run(dim, 32, 2, group, [20011, 9000], [new, new], causal=False, window=window, seed=9, every=range, max_len=20000)


def test_tiles_of_128_rows_with_pages_outside_the_cache():
    _run(128, 16, 32, 8, [300, 70, 700, 257], [64, 70, 65, 57], cut=[(0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (1, 4), (2, 43)])
    _run(256, 32, 32, 2, [300, 240], [75, 60], cut=[(0, 9), (1, 0)], causal=False)


@pytest.mark.parametrize("n", [65, 300, 4100])
def test_many_sequences(n):
    """More of them than one search step of 64 finds, some without rows, tokens or both."""
    rng = np.random.RandomState(n)
    lens = [int(x) for x in rng.randint(0, 50, n)]
    counts = [int(min(l, c)) for l, c in zip(lens, rng.randint(0, 5, n))]
    counts[-1], lens[-1] = 2, 40
    _run(64, 16, 2, 3, lens, counts, seed=n, heads=[1], every=range)


@pytest.mark.parametrize("n", [65, 4100])
@pytest.mark.parametrize("rows_each", [1, 12])
def test_append_of_many_sequences(n, rows_each):
    rng = np.random.RandomState(n)
    counts = [int(x) for x in rng.randint(0, 2 * rows_each + 1, n)]
    counts[0] += max(0, 8 * n + 1 - sum(counts)) if rows_each > 8 else 0
    lens = [c + int(x) for c, x in zip(counts, rng.randint(0, 20, n))]
    width = -(-max(lens) // 16)
    gen = torch.Generator("cuda").manual_seed(n)
    cache = _cache(gen, n * width, 1, 16, 64)
    table = torch.randperm(n * width, generator=gen, device="cuda").view(n, width)
    rows = sum(counts)
    k, v = (torch.randn(rows + 3, 1, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    want = OA.Cache.from_bytes(cache.k.cpu().numpy(), cache.v.cpu().numpy(), cache.k_scale.cpu().double().numpy(),
                               cache.v_scale.cpu().double().numpy(), 16)
    want.append(table.cpu().numpy(), [l - c for l, c in zip(lens, counts)], counts, k[:rows].double().cpu().numpy(),
                v[:rows].double().cpu().numpy())
    A.kv_append(cache, A.Batch(table.int(), _i32(lens), _i32(_cu(counts)), rows=rows + 3), k, v)
    _same_cache(cache, want)


@pytest.mark.parametrize("dim,hkv,group,n,length", [(128, 2, 24, 5, 300), (64, 1, 40, 3, 50), (256, 2, 17, 3, 90),
                                                    (64, 4, 2, 100, 260), (128, 8, 4, 40, 330), (64, 1, 1024, 1, 40),
                                                    (128, 1, 200, 2, 1500)])
def test_one_row_each_without_cu_rows(dim, hkv, group, n, length):
    """Query heads of a key head over one, several and many tiles; more
    workgroups than compute units."""
    _run(dim, 32, hkv, group, [max(1, length - 7 * i) for i in range(n)], [1] * n, cu=False)


def test_sequences_that_share_pages():
    _run(128, 32, 2, 4, [100, 64, 33], [1, 30, 2], shared=True, every=range)


def test_a_sequence_far_longer_than_stated():
    """200000 tokens where the host states 100: one workgroup takes them all."""
    _run(64, 128, 1, 2, [200000, 10], [2, 1], max_len=100, every=range)
    _run(256, 64, 1, 2, [100000], [3], max_len=100, every=range)


def test_two_captured_steps_share_a_workspace():
    """Replayed in turn with new lengths and row offsets, eager work between."""
    gen = torch.Generator("cuda").manual_seed(2)
    dim, page, hkv, group, width = 128, 16, 2, 4, 300
    cache = _cache(gen, 3 * width, hkv, page, dim)
    table = torch.randperm(3 * width, generator=gen, device="cuda").view(3, width).int()
    q = [torch.randn(8, hkv * group, dim, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    out = [torch.empty_like(x) for x in q]
    lens, cu = _i32([4000, 20, 900]), _i32([0, 1, 3, 6])
    batches = [A.Batch(table, lens, cu, rows=8, max_len=width * page) for _ in range(2)]
    need = batches[0].workspace_bytes(cache, hkv * group)
    assert need > 0
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for x, y, b in zip(q, out, batches):
        A.attention(x, cache, b, out=y, workspace=space)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            A.attention(x, cache, b, out=y, workspace=space)
        graphs.append(g)
    for step, (l, c) in enumerate([([4000, 20, 900], [0, 1, 3, 6]), ([4800, 0, 901], [0, 2, 2, 8]),
                                   ([3, 2500, 4700], [0, 0, 4, 5]), ([0, 0, 1], [0, 0, 0, 1])]):
        lens.copy_(_i32(l)), cu.copy_(_i32(c))
        for x, y in zip(q, out):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda")), y.fill_(7.0)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        for x, y in zip(q, out):
            want = torch.full_like(y, 7.0)
            A.attention(x, cache, A.Batch(table, _i32(l), _i32(c), rows=8, max_len=width * page), out=want)
            assert torch.equal(y, want), step


@pytest.mark.parametrize("dim,page,heads,rot,interleaved", [
    (128, 32, 3, 48, False), (128, 16, 5, 80, True), (64, 128, 2, 16, False), (256, 16, 2, 240, False),
    (256, 64, 3, 112, True), (128, 128, 2, 96, False), (64, 16, 9, 64, True)])
@pytest.mark.parametrize("static", [None, 0.25])
def test_append_of_many_rows_at_given_positions(dim, page, heads, rot, interleaved, static):
    """Positions that jump, run on, repeat and fall within a page; odd rotations;
    codes of normed keys are those of one rounding also with a static scale of a power of two."""
    log("append at positions %s" % ((dim, page, heads, rot, interleaved, static),))
    rng = np.random.RandomState(dim + page + rot)
    gen = torch.Generator("cuda").manual_seed(dim + page + rot)
    lens, counts = [3 * page + 5, 2 * page, page + 1], [2 * page + 9, 2 * page, page - 3]
    rows, width = sum(counts), 4
    table = torch.randperm(3 * width, generator=gen, device="cuda").view(3, width)
    cache = _cache(gen, 3 * width, heads, page, dim)
    if static:
        cache.k_scale.fill_(static), cache.v_scale.fill_(static)
    pos = np.arange(rows) + 1000
    jump = rng.rand(rows) < 0.2
    pos[jump] = rng.randint(0, 2 ** 24, jump.sum())
    pos[5] = pos[4]
    pos[8:11] = [2 ** 24, 2 ** 24 + 1, 0]
    freq = (1e5 ** (-torch.arange(rot // 2).double() / (rot // 2))).float()
    gamma = (1 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(torch.bfloat16)
    k, v = (torch.randn(rows, heads, dim, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    want = OA.Cache.from_bytes(cache.k.cpu().numpy(), cache.v.cpu().numpy(), cache.k_scale.cpu().double().numpy(),
                               cache.v_scale.cpu().double().numpy(), page)
    want.append(table.cpu().numpy(), [l - c for l, c in zip(lens, counts)], counts,
                OA.norm_rope(k.double().cpu().numpy(), gamma.double().cpu().numpy(), 1e-6, pos, freq.numpy(), interleaved),
                v.double().cpu().numpy(), static=static is not None)
    A.kv_append(cache, A.Batch(table.int(), _i32(lens), _i32(_cu(counts)), rows=rows), k, v, gamma, 1e-6,
                A.Rope(freq.cuda(), interleaved), _i32(pos.tolist()), static=static is not None)
    _same_cache(cache, want)


@pytest.mark.parametrize("rows_each", [2, 30])
def test_append_static_scales_that_are_no_powers_of_two(rows_each):
    gen = torch.Generator("cuda").manual_seed(rows_each)
    cache = _cache(gen, 8, 2, 32, 128, powers=False)
    cache.k_scale.mul_(20), cache.v_scale.mul_(20)
    want = OA.Cache.from_bytes(cache.k.cpu().numpy(), cache.v.cpu().numpy(), cache.k_scale.cpu().double().numpy(),
                               cache.v_scale.cpu().double().numpy(), 32)
    table = torch.arange(8, device="cuda").view(2, 4)
    k, v = ((20 * torch.randn(2 * rows_each, 2, 128, generator=gen, device="cuda")).to(torch.bfloat16) for _ in range(2))
    want.append(table.cpu().numpy(), [20, 40], [rows_each] * 2, k.double().cpu().numpy(), v.double().cpu().numpy(), static=True)
    A.kv_append(cache, A.Batch(table.int(), _i32([20 + rows_each, 40 + rows_each]), _i32([0, rows_each, 2 * rows_each]),
                               rows=2 * rows_each), k, v, static=True)
    _same_cache(cache, want)


def test_calls_on_another_stream_than_the_tensors_own():
    """The three calls handed a side stream, on tensors made on the current one."""
    gen = torch.Generator("cuda").manual_seed(1)
    cache = _cache(gen, 40, 2, 16, 64)
    twin = A.KVCache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone(), 16)
    table, lens = torch.arange(40, device="cuda").view(2, 20).int(), _i32([300, 17])
    x = [torch.randn(2, h, 64, generator=gen, device="cuda").to(torch.bfloat16) for h in (8, 2, 2)]
    rope, pos = A.Rope(torch.full((32,), 0.1, device="cuda")), _i32([299, 16])
    side = torch.cuda.Stream()

    def run(c, stream):
        b = A.Batch(table, lens)
        q, k = A.qk_norm_rope(x[0], x[1], pos, rope, stream=stream)
        A.kv_append(c, b, k, x[2], stream=stream)
        return (q, k) + A.attention(q, c, b, return_lse=True, stream=stream)

    want = run(cache, None)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = run(twin, stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(twin.k, cache.k) and torch.equal(twin.v, cache.v)


@pytest.mark.parametrize("dim,page,singles,long", [(128, 32, 30, 70), (64, 128, 30, 90), (256, 16, 9, 30), (128, 16, 3, 100)])
def test_append_of_a_prompt_among_single_tokens(dim, page, singles, long):
    """Both sides of the rule that picks a form by the average; the prompt begins within a page."""
    gen = torch.Generator("cuda").manual_seed(dim + page)
    counts = [1] * singles + [long]
    lens = [1 + 7 * i % 50 for i in range(singles)] + [long + 5]
    width = -(-max(lens) // page)
    n = singles + 1
    cache = _cache(gen, n * width, 3, page, dim)
    table = torch.randperm(n * width, generator=gen, device="cuda").view(n, width)
    rows = sum(counts)
    k, v = (torch.randn(rows, 3, dim, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    v[-long // 2:] *= 64                                            # the held codes are brought along
    gamma, freq = torch.ones(dim, device="cuda").to(torch.bfloat16), (1e4 ** (-torch.arange(32).double() / 32)).float()
    starts = [l - c for l, c in zip(lens, counts)]
    pos = np.concatenate([np.arange(s, s + c) for s, c in zip(starts, counts)])
    want = OA.Cache.from_bytes(cache.k.cpu().numpy(), cache.v.cpu().numpy(), cache.k_scale.cpu().double().numpy(),
                               cache.v_scale.cpu().double().numpy(), page)
    want.append(table.cpu().numpy(), starts, counts,
                OA.norm_rope(k.double().cpu().numpy(), np.ones(dim), 1e-6, pos, freq.numpy(), False), v.double().cpu().numpy())
    A.kv_append(cache, A.Batch(table.int(), _i32(lens), _i32(_cu(counts)), rows=rows), k, v, gamma, 1e-6, A.Rope(freq.cuda()))
    _same_cache(cache, want)


@pytest.mark.parametrize("dim,hkv,group,n,new", [(128, 2, 4, 2, 1), (64, 1, 40, 3, 2), (256, 2, 3, 2, 1), (128, 32, 8, 2, 128),
                                                 (256, 16, 4, 2, 70)])
@pytest.mark.parametrize("window", [1, 5, 100])
def test_lengths_far_behind_the_table_with_a_window(dim, hkv, group, n, new, window):
    """A length of 2^31 - 1 is cut to what the table holds, its rows keep their
    numbers and see nothing of it."""
    gen = torch.Generator("cuda").manual_seed(dim)
    cache = _cache(gen, 8, hkv, 16, dim)
    q = torch.randn(n * new, hkv * group, dim, generator=gen, device="cuda").to(torch.bfloat16)
    for lens in ([2 ** 31 - 1] * n, [2 ** 31 - 2 - 32 * i for i in range(n)], [2 ** 31 - 200] * n):
        batch = A.Batch(torch.arange(8, device="cuda").int().expand(n, 8).contiguous(), _i32(lens), _i32(_cu([new] * n)),
                        rows=n * new)
        y, lse = A.attention(q, cache, batch, window=window, out=torch.full_like(q, 7.0), return_lse=True)
        assert not y.any() and torch.isneginf(lse).all()
