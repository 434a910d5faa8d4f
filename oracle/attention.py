"""The attention between two W4A4 projections: norm and rotation of heads, a
paged 8-bit cache of keys and values (the paper serves its attention layers
with an FP8 KV cache, section 7 "KV-cache recipe"), and the attention over it.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Float64 throughout.

Readings: E4M3 is OCP E4M3FN; a page and head has one scale, the smallest power
of two s >= 2^-100 with amax <= 448 s over its tokens; a page written from its
first slot starts anew, a later write keeps the larger of its own scale and the
held one and re-rounds the held codes to it.
"""

import numpy as np

from .formats import E4M3_GRID, E4M3_MAX, e4m3_value, rne_index_sorted

E4M3_VALUES = np.array([e4m3_value(c) for c in range(256)], dtype=np.float64)
SCALE_FLOOR = 2.0 ** -100


def norm_rope(x, gamma, eps, positions, inv_freq, interleaved):
    """x [rows, heads, dim] float64; gamma [dim] or None; positions [rows]."""
    y = np.array(x, dtype=np.float64)
    if gamma is not None:
        mean = np.mean(y * y, axis=2, keepdims=True)
        y = y / np.sqrt(mean + float(np.float32(eps))) * gamma
    out = y.copy()
    half = 0 if inv_freq is None else len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * float(np.float32(inv_freq[i]))
        out[:, :, a] = y[:, :, a] * np.cos(angle) - y[:, :, b] * np.sin(angle)
        out[:, :, b] = y[:, :, b] * np.cos(angle) + y[:, :, a] * np.sin(angle)
    return out


def e4m3_codes(x):
    """Nearest E4M3 codes (ties to even), cut to 448, sign kept; 0x7F for NaN."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.where(np.isnan(x), 127, rne_index_sorted(np.abs(x), 1.0, E4M3_GRID))
    return np.where(np.signbit(x) & ~np.isnan(x), mag | 128, mag).astype(np.uint8)


def page_scale(amax):
    """The smallest power of two s >= 2^-100 with amax <= 448 s."""
    s = SCALE_FLOOR
    while amax > E4M3_MAX * s:
        s *= 2.0
    return s


def byte_places(page_size, dim, values):
    """[page_size, dim]: where a page's bytes hold token t's element e."""
    at = np.zeros((page_size, dim), dtype=np.int64)
    for t in range(page_size):
        for e in range(dim):
            u = t % 16
            if values:
                inside = (e // 64) * 1024 + (u // 4) * 256 + (e % 16) * 16 + (e // 16 % 4) * 4 + u % 4
            else:
                inside = (e // 16) * 256 + u * 16 + e % 16
            at[t, e] = (t // 16) * 16 * dim + inside
    return at


class Cache:
    """Codes [pages, heads, page_size, dim] uint8 and scales [pages, heads]."""

    def __init__(self, k, v, k_scale, v_scale):
        self.codes = [np.array(k), np.array(v)]
        self.scale = [np.array(k_scale, dtype=np.float64), np.array(v_scale, dtype=np.float64)]
        self.pages, self.heads, self.page_size, self.dim = self.codes[0].shape

    @classmethod
    def from_bytes(cls, k, v, k_scale, v_scale, page_size):
        """From the device order ([pages, heads, page_size * dim] bytes)."""
        dim = k.shape[2] // page_size
        return cls(k[:, :, byte_places(page_size, dim, False)], v[:, :, byte_places(page_size, dim, True)], k_scale,
                   v_scale)

    def to_bytes(self):
        out = []
        for values, codes in enumerate(self.codes):
            b = np.zeros((self.pages, self.heads, self.page_size * self.dim), dtype=np.uint8)
            b[:, :, byte_places(self.page_size, self.dim, bool(values))] = codes
            out.append(b)
        return out

    def append(self, table, starts, counts, k, v, static=False):
        """Rows of k, v [rows, heads, dim] in order: sequence b's counts[b] rows
        are its tokens from starts[b] on (tokens below 0 are dropped)."""
        row = 0
        for b, n in enumerate(counts):
            by_entry = {}
            for i in range(n):
                t = starts[b] + i
                if 0 <= t < table.shape[1] * self.page_size:
                    by_entry.setdefault(t // self.page_size, []).append((t % self.page_size, row + i))
            row += n
            for entry, tokens in by_entry.items():
                page = int(table[b, entry])
                if 0 <= page < self.pages:
                    self._append_page(page, tokens, (k, v), static)

    def _append_page(self, page, tokens, rows, static):
        slots, at = [s for s, _ in tokens], [r for _, r in tokens]
        for kind in (0, 1):
            for h in range(self.heads):
                x = rows[kind][at, h]
                s = self.scale[kind][page, h]
                if not static:
                    held, s = s, page_scale(np.abs(x).max())
                    if slots[0] > 0:
                        s = max(s, held)
                        old = E4M3_VALUES[self.codes[kind][page, h, :slots[0]]] * (held / s)
                        self.codes[kind][page, h, :slots[0]] = e4m3_codes(old)
                    self.scale[kind][page, h] = s
                self.codes[kind][page, h, slots] = e4m3_codes(x / s)

    def sequence(self, kind, pages, head, length):
        """(values [length, dim] with zeros for pages outside the cache, which
        tokens there are)."""
        x, there = np.zeros((length, self.dim)), np.zeros(length, dtype=bool)
        for t in range(length):
            page = int(pages[t // self.page_size])
            if 0 <= page < self.pages:
                x[t] = E4M3_VALUES[self.codes[kind][page, head, t % self.page_size]] * self.scale[kind][page, head]
                there[t] = True
        return x, there


def attention(q, cache, table, kv_len, counts, scale, causal, window):
    """y [rows, heads, dim], lse [rows, heads], and what bounds its error: the
    largest scale * sum_e |q_e k_e| of a seen token, sum_j p_j |v_j|, and the
    number of seen tokens times the largest |v| that their pages can hold."""
    rows, heads, dim = q.shape
    group = heads // cache.heads
    y, absolute = np.zeros_like(q), np.zeros_like(q)
    lse, size, most = np.full((rows, heads), -np.inf), np.zeros((rows, heads)), np.zeros((rows, heads))
    row = 0
    for b, n in enumerate(counts):
        length = min(max(int(kv_len[b]), 0), table.shape[1] * cache.page_size)
        for h in range(heads if n and length else 0):
            k, there = cache.sequence(0, table[b], h // group, length)
            v, _ = cache.sequence(1, table[b], h // group, length)
            for i in range(n):
                t = max(int(kv_len[b]), 0) - n + i
                j = np.arange(length)
                seen = there & ((j <= t) if causal else True) & ((j > t - window) if window > 0 else True)
                if not seen.any():
                    continue
                s = k[seen] @ q[row + i, h] * scale
                w = np.exp(s - s.max())
                y[row + i, h] = w @ v[seen] / w.sum()
                absolute[row + i, h] = w @ np.abs(v[seen]) / w.sum()
                lse[row + i, h] = s.max() + np.log(w.sum())
                held = [cache.scale[1][int(table[b, x // cache.page_size]), h // group] for x in np.flatnonzero(seen)]
                most[row + i, h] = len(held) * E4M3_MAX * max(held)
                size[row + i, h] = (np.abs(k[seen]) @ np.abs(q[row + i, h])).max() * abs(scale)
        row += n
    return y, lse, size, absolute, most
