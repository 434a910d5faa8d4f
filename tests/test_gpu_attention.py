"""GPU tests of the attention between two projections: norm and rotation,
append to the paged E4M3 cache, attention over it, against the float64 oracle.

Tolerances (before any run): a result rounded to bf16 is off by at most half a
step, 2^-8 of its value.  In front of that
  norm_rope   binary32 arithmetic, under ten roundings and a sine to 2^-22 on
              terms of at most |y_a| + |y_b|: 2^-20 of that;
  append      nothing: codes and scales are equal;
  attention   a probability is off by its rounding to binary16 (2^-11) and by
              its score's error, at most (head_dim + 4) 2^-24 of the largest
              scale * sum |q_e k_e|, twice (numerator and denominator), and
              2^-20 for the exponentials and sums; all of it on sum_j p_j |v_j|.
              Binary16 keeps 2^-25 below its normal range, of a probability times
              the value scale over the largest met: 2^-25 of the largest value
              that a page can hold (448 scales) for each token, over a sum of at
              least 1.  (Seen where one token takes all and holds zeros: y is
              then made of probabilities below 2^-14 alone.)
              A log-sum-exp is off by the score's error, 2^-20 and 2^-22 of itself.
"""

import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2609_04098_amd import attention as A
from paper_2609_04098_amd import linear as L
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def _bf16(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(torch.bfloat16)


def _np(t):
    return t.detach().cpu().double().numpy()


def _inv_freq(half, theta=1e4):
    return (theta ** (-torch.arange(half).double() / max(1, half))).float()


# ---------------------------------------------------------------- norm, rotation

@pytest.mark.parametrize("dim,rot,interleaved,hq,hk,rows,norm", [
    (128, 128, False, 5, 1, 3, True), (128, 128, True, 8, 8, 1, True), (128, 64, False, 40, 8, 17, True),
    (128, 16, True, 1, 0, 5, True), (128, 0, False, 3, 2, 7, True), (64, 64, False, 9, 3, 130, True),
    (64, 48, False, 0, 7, 33, True), (64, 32, True, 16, 1, 2, False), (256, 64, False, 6, 2, 41, True),
    (256, 256, False, 3, 1, 9, False), (256, 256, True, 17, 5, 4, True), (256, 80, False, 2, 2, 2100, True)])
def test_norm_rope(dim, rot, interleaved, hq, hk, rows, norm):
    log("norm_rope %s" % ((dim, rot, interleaved, hq, hk, rows, norm),))
    gen = torch.Generator().manual_seed(dim + rot + rows)
    qk = _bf16(gen, rows, (hq + hk) * dim + 24)                     # a fused projection with more columns
    gamma = [_bf16(gen, dim, scale=0.3) + 1 for _ in range(2)]
    pos = torch.randint(0, 2 ** 24, (rows,), generator=gen, dtype=torch.int32)
    pos[0] = 0
    freq = _inv_freq(rot // 2)
    dev = qk.cuda()
    q = dev[:, :hq * dim].view(rows, hq, dim) if hq else None
    k = dev[:, hq * dim:(hq + hk) * dim].view(rows, hk, dim) if hk else None
    g = [x.cuda() if norm else None for x in gamma]
    rope = A.Rope(freq.cuda(), interleaved)
    got = A.qk_norm_rope(q, k, pos.cuda(), rope, g[0], g[1], 1e-5)
    for x, y, gm in ((q, got[0], gamma[0]), (k, got[1], gamma[1])):
        if x is None:
            assert y is None
            continue
        want = OA.norm_rope(_np(x), _np(gm) if norm else None, 1e-5, pos.numpy(), freq.numpy() if rot else None,
                            interleaved)
        plain = OA.norm_rope(_np(x), _np(gm) if norm else None, 1e-5, pos.numpy(), None, interleaved)
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        size = np.abs(plain)
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
        bad = np.abs(_np(y) - want) > HALF * np.abs(want) + 2.0 ** -20 * size * (1 + HALF)
        assert not bad.any(), (bad.sum(), np.abs(_np(y) - want).max())
    if q is not None and k is not None:      # in place, and the columns behind are left
        tail = dev[:, (hq + hk) * dim:].clone()
        A.qk_norm_rope(q, k, pos.cuda(), rope, g[0], g[1], 1e-5, q_out=q, k_out=k)
        assert torch.equal(q, got[0]) and torch.equal(k, got[1]) and torch.equal(dev[:, (hq + hk) * dim:], tail)


def test_norm_rope_edges():
    rope = A.Rope(_inv_freq(64).cuda())
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    gamma = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    x[1] = 3e38
    x[2] = 1e-38
    x[3, 0, 7] = float("nan")
    q, _ = A.qk_norm_rope(x, None, pos, rope, gamma, eps=1e-6)
    assert not q[0].any() and torch.isnan(q[3, 0]).all() and not torch.isnan(q[3, 1]).any()
    y, _ = A.qk_norm_rope(x, None, pos, rope)           # no norm, position 0: the same values
    assert torch.equal(y[:3], x[:3])
    e, _ = A.qk_norm_rope(x[:0], None, pos[:0], rope, gamma)
    assert e.shape == (0, 2, 128)


# ---------------------------------------------------------------- the cache

def _random_cache(gen, pages, heads, page, dim, nan=True):
    """Random codes everywhere (NaN among them) and scales of all sizes."""
    codes = [torch.randint(0, 256, (pages, heads, page * dim), generator=gen, dtype=torch.int32).to(torch.uint8)
             for _ in range(2)]
    if not nan:
        codes = [torch.where((c & 127) == 127, c - 1, c) for c in codes]
    scales = [2.0 ** torch.randint(-12, -5, (pages, heads), generator=gen).float() for _ in range(2)]
    return A.KVCache(*[c.cuda() for c in codes], *[s.cuda() for s in scales], page)


def _oracle(cache):
    return OA.Cache.from_bytes(cache.k.cpu().numpy(), cache.v.cpu().numpy(), _np(cache.k_scale), _np(cache.v_scale),
                               cache.page_size)


def _same_cache(cache, want, what=""):
    k, v = want.to_bytes()
    assert np.array_equal(_np(cache.k_scale), want.scale[0]), what + ": key scales"
    assert np.array_equal(_np(cache.v_scale), want.scale[1]), what + ": value scales"
    for name, got, ref in (("keys", cache.k, k), ("values", cache.v, v)):
        got = got.cpu().numpy()
        bad = (got != ref) & ~(((got & 127) == 127) & ((ref & 127) == 127))      # (NaN has two codes)
        assert not bad.any(), "%s: %s, %d codes of %d" % (what, name, bad.sum(), bad.size)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(counts):
    return [0] + list(np.cumsum(counts))


@pytest.mark.parametrize("dim,page,heads,rot,interleaved,lens,counts", [
    (128, 16, 2, 128, False, [5, 16, 33, 0, 17], [5, 16, 20, 0, 1]),        # page ends, an empty sequence
    (128, 128, 1, 64, True, [130, 128, 1], [130, 1, 1]),
    (64, 32, 3, 64, False, [100, 7], [1, 7]),
    (64, 16, 1, 0, False, [40], [40]),
    (64, 128, 2, 32, False, [300, 129], [171, 3]),
    (256, 64, 2, 64, False, [70, 64, 200], [70, 2, 65]),
    (256, 16, 1, 256, True, [18, 16], [2, 16]),
    (256, 32, 4, 256, False, [33], [1])])
@pytest.mark.parametrize("norm", [True, False])
def test_append(dim, page, heads, rot, interleaved, lens, counts, norm):
    log("append %s" % ((dim, page, heads, rot, interleaved, lens, counts, norm),))
    gen = torch.Generator().manual_seed(dim + page + rot)
    width = max(-(-n // page) for n in lens) + 1
    table = torch.randperm(len(lens) * width + 2, generator=gen)[:len(lens) * width].view(len(lens), width)
    cache = _random_cache(gen, len(lens) * width + 2, heads, page, dim)
    rows = sum(counts)
    kv = _bf16(gen, rows + 2, 2 * heads * dim + 8)                  # two rows behind the last sequence
    kv[:, heads * dim:] *= torch.exp(torch.randn(rows + 2, 1, generator=gen) * 3).to(torch.bfloat16)
    gamma = (_bf16(gen, dim, scale=0.3) + 1) if norm else None
    freq = _inv_freq(rot // 2, 1e6)
    pos = None if counts[0] != 1 else torch.randint(0, 10 ** 6, (rows + 2,), generator=gen, dtype=torch.int32)
    want = _oracle(cache)
    starts = [n - c for n, c in zip(lens, counts)]
    own = np.concatenate([np.arange(s, s + c) for s, c in zip(starts, counts)]) if pos is None else pos.numpy()[:rows]
    k, v = kv[:, :heads * dim].view(-1, heads, dim), kv[:, heads * dim:2 * heads * dim].view(-1, heads, dim)
    want.append(table.numpy(), starts, counts,
                OA.norm_rope(_np(k[:rows]), None if gamma is None else _np(gamma), 1e-6, own,
                             freq.numpy() if rot else None, interleaved), _np(v[:rows]))
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=rows + 2)
    kvd = kv.cuda()
    kd, vd = kvd[:, :heads * dim].view(-1, heads, dim), kvd[:, heads * dim:2 * heads * dim].view(-1, heads, dim)
    A.kv_append(cache, batch, kd, vd, None if gamma is None else gamma.cuda(), 1e-6, A.Rope(freq.cuda(), interleaved),
                None if pos is None else pos.cuda())
    _same_cache(cache, want)
    A.kv_append(cache, batch, kd, vd, None if gamma is None else gamma.cuda(), 1e-6, A.Rope(freq.cuda(), interleaved),
                None if pos is None else pos.cuda())
    _same_cache(cache, want, "the same step again")


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 64)])
def test_append_token_by_token_and_growth(dim, page):
    """Tokens of all sizes, one a step, one row a sequence without cu_rows."""
    gen = torch.Generator().manual_seed(page)
    cache = _random_cache(gen, 9, 2, page, dim)
    want = _oracle(cache)
    table = torch.tensor([[4, 1], [0, 8], [6, 3]])
    for step in range(page + 3):
        x = _bf16(gen, 3, 2, dim) * float(2.0 ** ((step * 7) % 12 - 6))
        v = _bf16(gen, 3, 2, dim) * float(2.0 ** ((step * 5) % 9))
        if step == 4:
            x, v = x * 0, v * 0
        lens = [step + 1, step + 1, 0 if step % 2 else page]          # (the third: nothing, or its first page's last slot)
        want.append(table.numpy(), [n - 1 for n in lens], [1, 1, 1], _np(x), _np(v))
        A.kv_append(cache, A.Batch(table.int().cuda(), _i32(lens)), x.cuda(), v.cuda())
        _same_cache(cache, want, "step %d" % step)


def test_append_zeros_ties_and_extremes():
    """Exact ties of the rounding, zeros, both signs, the largest and smallest bf16 values."""
    dim, page = 64, 16
    cache = _random_cache(torch.Generator().manual_seed(0), 4, 1, page, dim)
    want = _oracle(cache)
    k = torch.zeros(4 * page, 1, dim)
    k[0, 0, 0] = 448
    k[0, 0, 1:] = torch.arange(63) * 0.5 - 15.75            # ties in the coarser binades
    k[1, 0] = (torch.arange(64) - 32) * 2.0 ** -10          # subnormal codes and their ties
    k[page] = 3.3e38                                        # a page of the largest values
    k[2 * page] = 1e-38                                     # and one below the smallest scale
    v = -k.flip(0)
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    table = torch.tensor([[2, 0, 3, 1]])
    want.append(table.numpy(), [0], [4 * page], _np(k), _np(v))
    A.kv_append(cache, A.Batch(table.int().cuda(), _i32([4 * page]), _i32([0, 4 * page]), rows=4 * page), k.cuda(), v.cuda())
    _same_cache(cache, want)


def test_append_values_next_to_a_border():
    """Normed keys within 2^-30 of a border between two codes: decided in 64 bits."""
    dim, page, n = 128, 16, 512
    gen = torch.Generator().manual_seed(8)
    k = torch.zeros(n, 1, dim)
    k[:, 0, 0] = 1.0                                                        # the others are much smaller
    k[:, 0, 1:] = torch.exp2(torch.randint(-12, -4, (n, dim - 1), generator=gen).float()) * \
        (1 + torch.randint(0, 128, (n, dim - 1), generator=gen) / 128)
    k = k.to(torch.bfloat16)
    gamma = (1 + torch.randint(0, 16, (dim,), generator=gen) / 16).to(torch.bfloat16)
    cache = _random_cache(gen, n // page, 1, page, dim)
    want = _oracle(cache)
    table = torch.arange(n // page)[None]
    want.append(table.numpy(), [0], [n], OA.norm_rope(_np(k), _np(gamma), 0.0, None, None, False), _np(k))
    A.kv_append(cache, A.Batch(table.int().cuda(), _i32([n]), _i32([0, n]), rows=n), k.cuda(), k.cuda(), gamma.cuda(), 0.0)
    _same_cache(cache, want)


def test_append_static_scales():
    gen = torch.Generator().manual_seed(3)
    dim, page = 128, 32
    cache = A.alloc_kv_cache(5, 2, dim, page, "cuda", scale=0.25)
    cache.k.zero_(), cache.v.zero_()
    want = _oracle(cache)
    k, v = _bf16(gen, 50, 2, dim), _bf16(gen, 50, 2, dim, scale=100.0)      # values over 448 * 0.25
    table = torch.tensor([[1, 4], [2, 0]])
    want.append(table.numpy(), [0, 3], [20, 30], _np(k), _np(v), static=True)
    A.kv_append(cache, A.Batch(table.int().cuda(), _i32([20, 33]), _i32([0, 20, 50]), rows=50), k.cuda(), v.cuda(),
                static=True)
    _same_cache(cache, want)


def test_append_out_of_bounds_inputs_write_nothing_else():
    """Pages outside the cache, tokens before 0 or behind the table, rows that
    cu_rows puts outside: dropped."""
    gen = torch.Generator().manual_seed(4)
    dim, page = 64, 16
    cache = _random_cache(gen, 6, 1, page, dim)
    want = _oracle(cache)
    table = torch.tensor([[-1, 3], [6, 2 ** 31 - 1], [5, 0], [1, 4]])
    lens, counts = [20, 25, 3, 40], [20, 25, 9, 20]         # the third has tokens before 0, the last ones behind the table
    k, v = _bf16(gen, 74, 1, dim), _bf16(gen, 74, 1, dim)
    want.append(table.numpy(), [n - c for n, c in zip(lens, counts)], counts, _np(k), _np(v))
    A.kv_append(cache, A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=74), k.cuda(), v.cuda())
    _same_cache(cache, want)
    for cu in ([0, -5, 90, 200, 74], [0, 100, 100, 100, 100]):
        guard = [torch.full((74, 1, dim), 1.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        A.kv_append(cache, A.Batch(table.int().cuda(), _i32([-7, 2 ** 31 - 1, 0, 16]), _i32(cu), rows=74), *guard)
    torch.cuda.synchronize()


# ---------------------------------------------------------------- attention

def _check(y, lse, cache, q, table, lens, counts, scale, causal, window):
    ref = OA.attention(_np(q), _oracle(cache), table.numpy(), lens, counts, scale, causal, window)
    want, want_lse, size, absolute, most = ref
    score = (cache.head_dim + 4) * 2.0 ** -24 * size
    before = absolute * (2.0 ** -11 + 2 * score[..., None] + 2.0 ** -20) + 2.0 ** -25 * most[..., None]
    rows = want.shape[0]
    err = np.abs(_np(y)[:rows] - want)
    bad = ~(err <= before + HALF * (np.abs(want) + before))
    assert not bad.any(), (bad.sum(), bad.size, float(np.nanmax(err)))
    if lse is not None:
        got = _np(lse)[:rows]
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got), empty)
        fine = ~empty
        got, want_lse, score = got[fine], want_lse[fine], score[fine]
        assert np.all(np.abs(got - want_lse) <= score + 2.0 ** -20 + 2.0 ** -22 * np.abs(want_lse))
        assert not _np(y)[:rows][empty].any()


def _attention_case(dim, page, hkv, group, lens, counts, causal, window, seed, cut=None, scale=None, max_len=None):
    gen = torch.Generator().manual_seed(seed)
    width = max(1, max(-(-n // page) for n in lens))
    n_pages = len(lens) * width + 2
    table = torch.randperm(n_pages, generator=gen)[:len(lens) * width].view(len(lens), width).clone()
    if cut is not None:
        table[cut] = n_pages + 5
    cache = _random_cache(gen, n_pages, hkv, page, dim)
    # No NaN among the tokens that the sequences hold; behind them there are.
    oracle = _oracle(cache)
    for b, n in enumerate(lens):
        for t in range(n):
            p = int(table[b, t // page])
            if p < n_pages:
                for c in oracle.codes:
                    x = c[p, :, t % page]
                    x[(x & 127) == 127] ^= 1
    for to, src in zip((cache.k, cache.v), oracle.to_bytes()):
        to.copy_(torch.from_numpy(src))
    rows = sum(counts)
    q = _bf16(gen, rows + 3, hkv * group * dim + 8, scale=0.5)
    qd = q.cuda()[:, :hkv * group * dim].view(rows + 3, hkv * group, dim)
    out = torch.full((rows + 3, hkv * group * dim + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    y = out[:, 8:hkv * group * dim + 8].view(rows + 3, hkv * group, dim)
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=rows + 3, max_len=max_len)
    scale = dim ** -0.5 if scale is None else scale
    got, lse = A.attention(qd, cache, batch, scale=scale, causal=causal, window=window, out=y, return_lse=True)
    assert got is y
    _check(y, lse, cache, qd[:rows], table, lens, counts, scale, causal, window)
    out[:rows, 8:hkv * group * dim + 8] = 7.0           # rows behind the last sequence, columns around: left
    assert torch.equal(out, torch.full_like(out, 7.0))


CASES = [
    # dim, page, key heads, group, lengths, new rows
    (128, 16, 2, 4, [1, 17, 300, 64], [1, 1, 1, 1]),
    (128, 32, 1, 5, [33, 0, 5, 70], [3, 2, 5, 0]),              # no tokens, no rows
    (128, 64, 2, 1, [90, 31], [40, 31]),
    (128, 128, 1, 16, [257], [2]),
    (128, 16, 1, 7, [200, 90], [120, 90]),
    (64, 16, 3, 2, [40, 100, 16], [16, 1, 16]),
    (64, 128, 1, 33, [129, 3], [1, 3]),
    (64, 32, 2, 8, [600], [9]),
    (256, 16, 1, 6, [50, 20], [2, 20]),
    (256, 64, 2, 3, [140, 65], [1, 65]),
    (256, 32, 1, 24, [31], [31]),
]


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 20), (False, 33), (True, 1)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "d%d_p%d_h%dx%d" % c[:4])
def test_attention(case, causal, window):
    log("attention %s causal %s window %d" % (case, causal, window))
    _attention_case(*case, causal, window, seed=case[0] + case[1] + window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_of_long_sequences_in_pieces(dim):
    """Few rows: the tokens are divided; and the same with a length that the
    host states too low or not at all."""
    for max_len in (None, 2600, 100, 1500):
        log("pieces, dim %d, max_len %s" % (dim, max_len))
        _attention_case(dim, 32, 1, 4, [2600, 1, 900], [1, 1, 2], True, 0, seed=dim, max_len=max_len)
    _attention_case(dim, 16, 2, 3, [2100, 1200], [3, 40], True, 1000, seed=dim + 1)
    _attention_case(dim, 16, 2, 3, [0, 2100], [3, 2], False, 500, seed=dim + 2)


@pytest.mark.parametrize("counts", [[1, 1, 1], [40, 30, 20]])
def test_attention_masks_pages_outside_the_cache(counts):
    _attention_case(128, 16, 1, 4, [100, 50, 20], counts, True, 0, seed=1, cut=(0, 2))
    _attention_case(64, 32, 1, 4, [100, 50, 20], counts, True, 0, seed=2, cut=(slice(None), 0))


@pytest.mark.parametrize("scale", [0.0, -0.2, 30.0])
def test_attention_scales(scale):
    """No preference, the opposite one, and one token that takes all."""
    _attention_case(128, 32, 1, 4, [100, 50], [1, 50], True, 0, seed=5, scale=scale)


@pytest.mark.parametrize("counts", [[1, 1], [90, 64]])
def test_attention_values_of_very_different_pages(counts):
    """Value scales from 2^-100 to 2^20: the binary16 products lose nothing of weight."""
    gen = torch.Generator().manual_seed(6)
    cache = _random_cache(gen, 12, 1, 16, 128, nan=False)
    cache.v_scale.copy_(2.0 ** torch.tensor([-100, 20, -8, 5, -30, 0, 15, -100, -3, 11, 2, -20.0])[:, None])
    table = torch.randperm(12, generator=gen).view(2, 6)
    lens = [90, 70]
    q = _bf16(gen, sum(counts), 4, 128)
    batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=sum(counts))
    y, lse = A.attention(q.cuda(), cache, batch, return_lse=True)
    _check(y, lse, cache, q, table, lens, counts, 128 ** -0.5, True, 0)


def test_attention_nan_reaches_only_the_rows_that_see_it():
    gen = torch.Generator().manual_seed(7)
    cache = _random_cache(gen, 4, 1, 16, 64, nan=False)
    q = _bf16(gen, 60, 2, 64).cuda()
    batch = A.Batch(_i32([[2, 0, 3, 1]]), _i32([60]), _i32([0, 60]), rows=60)
    clean = A.attention(q, cache, batch)
    cache.k[0, 0, 8 * 16] = 0x7F                       # token 16 + 8, element 0
    y, lse = A.attention(q, cache, batch, return_lse=True)
    assert torch.equal(y[:24], clean[:24]) and torch.isnan(y[24:]).all() and torch.isnan(lse[24:]).all()
    q[3] = float("nan")                                # a row of its own
    y2 = A.attention(q, cache, batch)
    assert torch.isnan(y2[3]).all() and torch.equal(y2[:3], y[:3]) and torch.equal(y2[4:24], y[4:24])


def test_attention_of_malformed_device_values_stays_inside():
    """Lengths and row offsets that make no sense: nothing outside the tensors
    is touched (canaries around the output), rows that no sequence has are left."""
    gen = torch.Generator().manual_seed(9)
    cache = _random_cache(gen, 4, 1, 16, 64, nan=False)
    q = _bf16(gen, 20, 2, 64).cuda()
    out = torch.full((24, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for lens, cu in (([-5, 2 ** 31 - 1], [0, 10, 20]), ([40, 50], [5, -3, 1000]), ([64, 64], [0, 20, 3])):
        A.attention(q, cache, A.Batch(_i32([[0, 1, 2, 3], [3, 2, 1, 0]]), _i32(lens), _i32(cu), rows=20), out=out[2:22])
    assert (out[:2] == 7).all() and (out[22:] == 7).all()


def test_far_pages_of_a_large_cache():
    """Page offsets over 2^32 bytes (a strided cache of 5 GiB)."""
    gen = torch.Generator().manual_seed(10)
    stride = 1 << 30
    buf = torch.empty(5 * stride, dtype=torch.uint8, device="cuda")
    k = torch.as_strided(buf, (5, 1, 16 * 128), (stride, 16 * 128, 1))
    v = torch.as_strided(buf, (5, 1, 16 * 128), (stride, 16 * 128, 1), storage_offset=stride // 2)
    cache = A.KVCache(k, v, torch.zeros(5, 1, device="cuda"), torch.zeros(5, 1, device="cuda"), 16)
    batch = A.Batch(_i32([[4, 0, 3]]), _i32([40]), _i32([0, 40]), rows=40)
    x = [_bf16(gen, 40, 1, 128) for _ in range(2)]
    k.zero_(), v.zero_()
    want = _oracle(cache)
    want.append(np.array([[4, 0, 3]]), [0], [40], _np(x[0]), _np(x[1]))
    A.kv_append(cache, batch, x[0].cuda(), x[1].cuda())
    _same_cache(cache, want)
    q = _bf16(gen, 40, 4, 128).cuda()
    y, lse = A.attention(q, cache, batch, return_lse=True)
    _check(y, lse, cache, q, torch.tensor([[4, 0, 3]]), [40], [40], 128 ** -0.5, True, 0)


# ---------------------------------------------------------------- together

def _layer(x, w_qkv, w_out, gammas, rope, cache, batch, pos, hq, hkv, dim, stream=None):
    """One attention layer between its W4A4 projections."""
    qkv = L.gemm(L.quantize_act(x, stream=stream), w_qkv, stream=stream)
    n = qkv.shape[0]
    q = qkv[:, :hq * dim].view(n, hq, dim)
    k = qkv[:, hq * dim:(hq + hkv) * dim].view(n, hkv, dim)
    v = qkv[:, (hq + hkv) * dim:].view(n, hkv, dim)
    qr, _ = A.qk_norm_rope(q, None, pos, rope, gammas[0], stream=stream)
    A.kv_append(cache, batch, k, v, gammas[1], rope=rope, stream=stream)
    y = A.attention(qr, cache, batch, stream=stream)
    return qkv, qr, y, L.gemm(L.quantize_act(y.view(n, hq * dim), stream=stream), w_out, stream=stream)


def _layer_inputs(seed, hq, hkv, dim, hidden):
    gen = torch.Generator().manual_seed(seed)
    w = _bf16(gen, (hq + 2 * hkv) * dim, hidden, scale=0.05).cuda()
    seg = [0, hq * dim, (hq + hkv) * dim, (hq + 2 * hkv) * dim]
    return (gen, L.pack_weight(w, seg), L.pack_weight(_bf16(gen, hidden, hq * dim, scale=0.05).cuda()),
            [(_bf16(gen, dim, scale=0.2) + 1).cuda() for _ in range(2)], A.Rope(_inv_freq(dim // 4).cuda()))


def test_a_layer_prompt_then_tokens():
    """Prompt, then single tokens, each step against the oracle from the
    projection's own output on."""
    hq, hkv, dim, hidden, page = 8, 2, 128, 256, 32
    gen, w_qkv, w_out, gammas, rope = _layer_inputs(11, hq, hkv, dim, hidden)
    cache = A.alloc_kv_cache(8, hkv, dim, page, "cuda")
    cache.k.fill_(0x7F), cache.v.fill_(0x7F)
    want = _oracle(cache)
    table = torch.tensor([[5, 1, 7], [0, 6, 2]])
    lens = [0, 0]
    for counts in ([30, 45], [1, 1], [1, 1], [3, 1], [1, 0]):
        lens = [n + c for n, c in zip(lens, counts)]
        rows = sum(counts)
        x = _bf16(gen, rows, hidden).cuda()
        pos = np.concatenate([np.arange(n - c, n) for n, c in zip(lens, counts)])
        batch = A.Batch(table.int().cuda(), _i32(lens), _i32(_cu(counts)), rows=rows, max_len=max(lens))
        qkv, qr, y, z = _layer(x, w_qkv, w_out, gammas, rope, cache, batch, _i32(pos.tolist()), hq, hkv, dim)
        k = _np(qkv[:, hq * dim:(hq + hkv) * dim].reshape(rows, hkv, dim))
        v = _np(qkv[:, (hq + hkv) * dim:].reshape(rows, hkv, dim))
        want.append(table.numpy(), [n - c for n, c in zip(lens, counts)], counts,
                    OA.norm_rope(k, _np(gammas[1]), 1e-6, pos, rope.inv_freq.cpu().numpy(), False), v)
        _same_cache(cache, want, "lengths %s" % lens)
        _check(y, None, cache, qr, table, lens, counts, dim ** -0.5, True, 0)
        assert torch.isfinite(z).all() and z.shape == (rows, hidden)


def test_a_captured_step_replays_with_new_lengths():
    """Append and attention of one decode step in a graph, replayed while the
    lengths, the tokens and the eager work between the replays go on."""
    hq, hkv, dim, hidden, page = 8, 2, 128, 256, 16
    gen, w_qkv, w_out, gammas, rope = _layer_inputs(12, hq, hkv, dim, hidden)
    caches = [A.alloc_kv_cache(1262, hkv, dim, page, "cuda") for _ in range(2)]
    table = torch.randperm(1262, generator=gen)[:1260].view(3, 420).int().cuda()
    start = [4900, 40, 15]
    prompt = _bf16(gen, sum(start), hidden).cuda()
    lens, pos = _i32(start), _i32(start)
    ppos = _i32(np.concatenate([np.arange(n) for n in start]).tolist())
    x = torch.empty(3, hidden, dtype=torch.bfloat16, device="cuda")
    for c in caches:
        _layer(prompt, w_qkv, w_out, gammas, rope, c,
               A.Batch(table, lens.clone(), _i32(_cu(start)), rows=sum(start)), ppos, hq, hkv, dim)
    step = A.Batch(table, lens, max_len=420 * page)
    assert step.workspace_bytes(caches[0], hq) > 0
    lens += 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(x.zero_(), w_qkv, w_out, gammas, rope, caches[1], step, pos, hq, hkv, dim)      # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _layer(x, w_qkv, w_out, gammas, rope, caches[1], step, pos, hq, hkv, dim)
    for i in range(6):
        x.copy_(_bf16(gen, 3, hidden))
        graph.replay()
        want = _layer(x, w_qkv, w_out, gammas, rope, caches[0], A.Batch(table, lens.clone(), max_len=420 * page),
                      pos.clone(), hq, hkv, dim)
        for a, b in zip(got, want):
            assert torch.equal(a, b), "replay %d" % i
        lens += 1
        pos += 1
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Two layers on two streams, each with its own cache and workspace."""
    hq, hkv, dim, hidden, page = 8, 2, 64, 256, 16
    gen, w_qkv, w_out, gammas, rope = _layer_inputs(13, hq, hkv, dim, hidden)
    table, lens = torch.arange(264).view(2, 132).int().cuda(), [2000, 1990]
    x = _bf16(gen, 2, hidden).cuda()
    pos = _i32([n - 1 for n in lens])
    codes = [torch.randint(0, 100, (264, hkv, page * dim), generator=gen, dtype=torch.int32).to(torch.uint8).cuda()
             for _ in range(2)]
    scales = torch.full((264, hkv), 2.0 ** -6, device="cuda")

    def run(stream):
        cache = A.KVCache(codes[0].clone(), codes[1].clone(), scales.clone(), scales.clone(), page)
        batch = A.Batch(table, _i32(lens), max_len=2000)
        if stream is not None:
            torch.cuda.synchronize()
        out = [_layer(x, w_qkv, w_out, gammas, rope, cache, batch, pos, hq, hkv, dim, stream)[3] for _ in range(5)]
        return out, cache

    want, _ = run(None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [run(s) for s in streams]
    torch.cuda.synchronize()
    for out, _ in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_results_do_not_depend_on_the_run():
    gen = torch.Generator().manual_seed(14)
    cache = _random_cache(gen, 80, 2, 32, 128, nan=False)
    q = _bf16(gen, 45, 8, 128).cuda()
    batch = A.Batch(torch.arange(80).view(2, 40).int().cuda(), _i32([1270, 900]), _i32([0, 1, 45]), rows=45)
    first = A.attention(q, cache, batch, return_lse=True)
    for _ in range(5):
        again = A.attention(q, cache, batch, return_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
