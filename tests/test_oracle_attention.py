"""Pins of the attention oracle: closed forms of the norm, the rotation, the
page scales, the byte order and the softmax, and independent evaluations with
PyTorch in float64."""

import math

import numpy as np
import torch

from oracle import attention as OA


def test_norm_closed_forms():
    x = np.zeros((1, 2, 64))
    x[0, 0] = 3.0
    x[0, 1, 5] = -2.0
    gamma = np.linspace(0.5, 2, 64)
    y = OA.norm_rope(x, gamma, 0.0, [0], None, False)
    assert np.allclose(y[0, 0], gamma, rtol=1e-15)
    assert np.isclose(y[0, 1, 5], -8.0 * gamma[5], rtol=1e-15) and np.count_nonzero(y[0, 1]) == 1
    # eps inside the root: a constant head c with eps = c^2 gives gamma / sqrt 2
    y = OA.norm_rope(x[:, :1], gamma, 9.0, [0], None, False)
    assert np.allclose(y[0, 0], gamma / math.sqrt(2), rtol=1e-15)
    assert np.array_equal(OA.norm_rope(x, None, 0.0, [0], None, False), x)


def test_rotation_is_a_complex_product():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 64))
    pos = np.array([0, 1, 7, 100003, 16000000])
    freq = (1e4 ** -(np.arange(16) / 16)).astype(np.float32)
    for interleaved in (False, True):
        y = OA.norm_rope(x, None, 0.0, pos, freq, interleaved)
        a, b = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, None, None] * freq.astype(np.float64))
        assert np.allclose(y[..., a], z.real, atol=1e-9) and np.allclose(y[..., b], z.imag, atol=1e-9)
        assert np.array_equal(y[..., 32:], x[..., 32:]) and np.array_equal(y[0], x[0])


def test_codes_match_the_torch_cast():
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.standard_normal(4000) * np.exp(rng.uniform(-8, 5, 4000)), np.arange(-448, 449, 0.5),
                        np.arange(-64, 65) * 2.0 ** -11])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(OA.e4m3_codes(x), want)
    codes = np.arange(256)
    codes[255] = 0x7F                                    # (NaN has one code here; zeros keep their signs)
    assert np.array_equal(OA.e4m3_codes(OA.E4M3_VALUES), codes)
    assert OA.e4m3_codes([1e9])[0] == 0x7E and OA.e4m3_codes([-1e9])[0] == 0xFE
    values = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(OA.E4M3_VALUES, values, equal_nan=True)


def test_page_scale():
    for e in (-60, -3, 0, 5, 100):
        assert OA.page_scale(448 * 2.0 ** e) == 2.0 ** e
        assert OA.page_scale(np.nextafter(448 * 2.0 ** e, np.inf)) == 2.0 ** (e + 1)
    assert OA.page_scale(0.0) == OA.page_scale(1e-40) == 2.0 ** -100


def test_byte_order():
    for page, dim in ((16, 64), (32, 128), (64, 256)):
        for values in (False, True):
            at = OA.byte_places(page, dim, values)
            assert np.array_equal(np.sort(at.ravel()), np.arange(page * dim))
        k, v = OA.byte_places(page, dim, False), OA.byte_places(page, dim, True)
        # keys: 16 consecutive elements of a token, then the group's next token
        assert k[0, 0] == 0 and k[0, 15] == 15 and k[1, 0] == 16 and k[0, 16] == 256
        # values: 4 consecutive tokens of an element, then elements 16 apart, then the next element
        assert [v[t, 0] for t in range(4)] == [0, 1, 2, 3] and v[0, 16] == 4 and v[0, 1] == 16 and v[4, 0] == 256
        assert (k[15].max() < 16 * dim) and (v[15].max() < 16 * dim)
    rng = np.random.default_rng(3)
    c = OA.Cache(*[rng.integers(0, 256, (2, 2, 32, 64), dtype=np.uint8) for _ in range(2)], np.ones((2, 2)),
                 np.ones((2, 2)))
    back = OA.Cache.from_bytes(*c.to_bytes(), *c.scale, 32)
    assert all(np.array_equal(a, b) for a, b in zip(c.codes, back.codes))


def _empty(pages, heads, page, dim):
    z = np.full((pages, heads, page, dim), 0x7F, dtype=np.uint8)
    return OA.Cache(z, z, np.full((pages, heads), 123.0), np.full((pages, heads), 123.0))


def test_append_scales_grow_and_start_anew():
    c = _empty(3, 1, 16, 64)
    table = np.array([[2, 0]])
    x = np.zeros((20, 1, 64))
    x[:, 0, 0] = 1.0
    x[17, 0, 3] = 500.0
    c.append(table, [0], [15], x[:15], -x[:15])                 # tokens 0 .. 14
    assert c.scale[0][2, 0] == 2.0 ** -8 and c.scale[0][0, 0] == 123.0
    assert np.all(OA.E4M3_VALUES[c.codes[0][2, 0, :15, 0]] == 256) and c.codes[0][2, 0, 15, 0] == 0x7F
    c.append(table, [15], [3], x[15:18], -x[15:18])             # 15 in the first page, 16 and 17 in the second
    assert c.scale[0][2, 0] == 2.0 ** -8 and c.scale[0][0, 0] == 2.0
    assert OA.E4M3_VALUES[c.codes[1][0, 0, 1, 3]] == -256 and OA.E4M3_VALUES[c.codes[1][0, 0, 1, 0]] == -0.5
    c.append(table, [14], [1], 1e4 * x[:1], x[:1])              # the page's scale grows: held tokens follow
    assert c.scale[0][2, 0] == 32.0 and OA.E4M3_VALUES[c.codes[0][2, 0, 3, 0]] == 1 / 32
    assert c.scale[1][2, 0] == 2.0 ** -8                        # values did not grow
    c.append(table, [0], [1], x[:1], x[:1])                     # from slot 0: anew
    assert c.scale[0][2, 0] == 2.0 ** -8
    before = [a.copy() for a in c.codes]
    c.append(np.array([[7, -1]]), [0], [17], x[:17], x[:17])    # pages outside the cache
    c.append(table, [-4], [4], x[:4], x[:4])                    # tokens below 0
    assert all(np.array_equal(a, b) for a, b in zip(before, c.codes))


def test_append_static_keeps_scales_and_saturates():
    c = _empty(1, 1, 16, 64)
    x = np.linspace(-1e6, 1e6, 64).reshape(1, 1, 64)
    c.append(np.array([[0]]), [3], [1], x, x / 1e6, static=True)
    assert c.scale[0][0, 0] == 123.0
    assert c.codes[0][0, 0, 3, 0] == 0xFE and c.codes[0][0, 0, 3, 63] == 0x7E


def test_attention_against_torch_and_closed_forms():
    rng = np.random.default_rng(5)
    pages, heads, page, dim, group = 6, 2, 16, 64, 3
    code = rng.integers(0, 0x70, (2, pages, heads, page, dim)).astype(np.uint8) | \
        (rng.integers(0, 2, (2, pages, heads, page, dim)) * 128).astype(np.uint8)
    scale = 2.0 ** rng.integers(-9, -5, (2, pages, heads))
    c = OA.Cache(code[0], code[1], scale[0], scale[1])
    table = np.array([[3, 0, 5], [1, 2, 4]])
    q = rng.standard_normal((9, heads * group, dim))
    kv_len, counts = [41, 3], [5, 4]
    for causal, window in ((True, 0), (False, 0), (True, 7), (False, 7)):
        y, lse, _, _, _ = OA.attention(q, c, table, kv_len, counts, 0.3, causal, window)
        nat = [torch.from_numpy(OA.E4M3_VALUES[code[i]] * scale[i][:, :, None, None]) for i in (0, 1)]
        row = 0
        for b in range(2):
            k, v = [x[torch.from_numpy(table[b])].transpose(0, 1).reshape(heads, -1, dim)[:, :kv_len[b]]
                    .repeat_interleave(group, 0) for x in nat]
            x = torch.from_numpy(q[row:row + counts[b]]).transpose(0, 1)
            s = x @ k.transpose(1, 2) * 0.3
            t = kv_len[b] - counts[b] + torch.arange(counts[b])[:, None]
            j = torch.arange(kv_len[b])[None]
            hide = ((j > t) if causal else torch.zeros_like(j > t)) | ((j <= t - window) if window else (j < 0))
            s = s.masked_fill(hide, -math.inf)
            want = torch.softmax(s, -1) @ v
            empty = hide.all(-1)
            want[:, empty] = 0.0
            assert np.allclose(y[row:row + counts[b]], want.transpose(0, 1).numpy(), atol=1e-12)
            assert np.allclose(lse[row:row + counts[b]], torch.logsumexp(s, -1).T.numpy(), atol=1e-12)
            row += counts[b]
    # the first row of the second sequence (token -1) sees nothing under a causal mask
    y, lse, size, absolute, most = OA.attention(q, c, table, kv_len, counts, 0.3, True, 0)
    assert not y[5].any() and np.all(np.isneginf(lse[5]))
    # the row at token 0 sees only that one: y is its value, lse its score, and the bounds are those of one token
    k0, v0 = [OA.E4M3_VALUES[code[i][1, :, 0]] * scale[i][1][:, None] for i in (0, 1)]
    for h in range(heads * group):
        assert np.allclose(y[6, h], v0[h // group]) and np.isclose(lse[6, h], q[6, h] @ k0[h // group] * 0.3)
        assert np.isclose(size[6, h], np.abs(q[6, h] * k0[h // group]).sum() * 0.3)
        assert np.allclose(absolute[6, h], np.abs(v0[h // group]))
        assert most[6, h] == 448 * scale[1][1, h // group]
        assert most[8, h] == 3 * 448 * scale[1][1, h // group] and most[5, h] == 0
    # pages outside the cache are masked
    bad = table.copy()
    bad[0, 1] = 99
    y2 = OA.attention(q, c, bad, kv_len, counts, 0.3, True, 0)[0]
    keep = np.r_[0:16, 32:41]
    k, v = [np.concatenate([OA.E4M3_VALUES[code[i][p, 0]] * scale[i][p, 0] for p in (3, 0, 5)])[keep] for i in (0, 1)]
    s = np.exp(k @ q[4, 0] * 0.3)
    assert np.allclose(y2[4, 0], s @ v / s.sum())
