"""The attention between two W4A4 projections, on top of the C ABI
(include/nvfp4_attention.h): argument checks, buffers and call order only.

    rope  = Rope(inv_freq)                                # once
    cache = alloc_kv_cache(num_pages, kv_heads, head_dim, page_size, device)   # per layer
    batch = Batch(page_table, kv_len, cu_rows)            # per step, for all layers
    q, _  = qk_norm_rope(q, None, positions, rope, q_gamma)
    kv_append(cache, batch, k, v, k_gamma, rope=rope)     # E4M3, a scale for each page and head
    y     = attention(q, cache, batch)                    # softmax(q k' / sqrt(d)) v

q, k and v are bf16 [rows, heads, head_dim] views, as a fused projection's
output leaves them (heads side by side, any row stride that is a multiple of 8).
"""

import ctypes
import math

import torch

from . import linear as _l
from . import nvfp4 as _c
from . import nvfp4_attention as _a


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _rows_ok(x, heads, dim, name):
    """bf16 [rows, heads, dim], heads side by side."""
    _need(x.dtype == torch.bfloat16 and x.dim() == 3, "%s must be a bf16 [rows, heads, head_dim] tensor" % name)
    _need(x.shape[2] == dim and (heads is None or x.shape[1] == heads), "%s has the wrong heads or head_dim" % name)
    _need(x.numel() == 0 or (x.stride(2) == 1 and (x.shape[1] == 1 or x.stride(1) == dim)),
          "%s must have its heads side by side" % name)


def _like_rows(x, stream):
    """A contiguous [rows, heads, head_dim] tensor from the stream that uses it."""
    with _l._on(stream, x.device):
        return torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _on_device(t):
    """Context in which t's device is the current one (kernels are launched on
    the current device, on its current stream)."""
    if t.device.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    return torch.cuda.device(t.device)


def _run(t, call, *args):
    """``call(*args)`` with t's device current; no context where it is."""
    if t.is_cuda and t.get_device() == torch.cuda.current_device():
        return call(*args)
    with _on_device(t):
        return call(*args)


class Rope:
    """The rotation of a head's first 2 * len(inv_freq) elements by the angles
    position * inv_freq[i] (float32, on the GPU): element i with element
    i + len(inv_freq), or 2 i with 2 i + 1 if ``interleaved``."""

    def __init__(self, inv_freq, interleaved=False):
        _need(inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.shape[0] % 8 == 0,
              "inv_freq must be a float32 vector of a multiple of 8 elements")
        _need(not inv_freq.requires_grad, "inv_freq takes no gradient here")
        self.inv_freq = inv_freq.contiguous() if inv_freq.shape[0] else None
        self.interleaved = 1 if interleaved else 0


class KVCache:
    """A layer's paged cache over given buffers: k, v uint8 [num_pages,
    kv_heads, page_size * head_dim] in the order that nvfp4_attention.h states
    (any page stride that is a multiple of 16), k_scale, v_scale float32
    [num_pages, kv_heads] with one row stride."""

    def __init__(self, k, v, k_scale, v_scale, page_size):
        for name, t in (("k", k), ("v", v)):
            _need(t.dtype == torch.uint8 and t.dim() == 3 and t.shape == k.shape and t.shape[2] % page_size == 0,
                  "%s must be uint8 [num_pages, kv_heads, page_size * head_dim]" % name)
            _need(t.stride(2) == 1 and (t.shape[1] == 1 or t.stride(1) == t.shape[2]),
                  "the heads of a page of %s must be side by side" % name)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _need(t.dtype == torch.float32 and t.shape == k.shape[:2] and t.stride(0) == k_scale.stride(0)
                  and (t.shape[1] == 1 or t.stride(1) == 1), "%s must be float32 [num_pages, kv_heads]" % name)
        _need(k.device == v.device == k_scale.device == v_scale.device, "the cache's buffers are on several devices")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.page_size, self.kv_heads, self.head_dim = page_size, k.shape[1], k.shape[2] // page_size
        self.device = k.device
        self.struct = _a.cache_struct(k, v, k_scale, v_scale, page_size)
        self.ref = ctypes.byref(self.struct)

    def tokens(self):
        """(keys, values) as float32 [num_pages, kv_heads, page_size, head_dim]: every
        slot's code times its page's scale (for inspection)."""
        n, h, p, d = self.k.shape[0], self.kv_heads, self.page_size, self.head_dim
        k = self.k.reshape(n, h, p // 16, d // 16, 16, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, h, p, d)
        v = self.v.reshape(n, h, p // 16, d // 64, 4, 16, 4, 4).permute(0, 1, 2, 4, 7, 3, 6, 5).reshape(n, h, p, d)
        return (k.view(torch.float8_e4m3fn).float() * self.k_scale[:, :, None, None],
                v.view(torch.float8_e4m3fn).float() * self.v_scale[:, :, None, None])


def alloc_kv_cache(num_pages, kv_heads, head_dim, page_size, device, scale=None):
    """An empty cache; with ``scale`` every page's scale is set to it (for
    ``kv_append(..., static=True)``)."""
    codes = [torch.empty((num_pages, kv_heads, page_size * head_dim), dtype=torch.uint8, device=device)
             for _ in range(2)]
    scales = [torch.full((num_pages, kv_heads), 0.0 if scale is None else float(scale), dtype=torch.float32,
                         device=device) for _ in range(2)]
    return KVCache(*codes, *scales, page_size)


class Batch:
    """A step's sequences: page_table int32 [n_seqs, max_pages], kv_len int32
    [n_seqs] (tokens with the new ones), cu_rows int32 [n_seqs + 1] (None: one
    new row for each sequence), all on the GPU.  ``rows``: rows of the step's
    tensors (needed with cu_rows, whose values stay on the GPU).  ``max_len``:
    the largest kv_len as far as the host knows it (else what the page table
    can hold, for pages of ``page_size`` tokens at most 128); work is divided
    by it, so that a tight value is faster."""

    def __init__(self, page_table, kv_len, cu_rows=None, rows=None, max_len=None):
        _need(page_table.dtype == torch.int32 and page_table.dim() == 2
              and (page_table.shape[1] <= 1 or page_table.stride(1) == 1), "page_table must be int32 [n_seqs, max_pages]")
        n = page_table.shape[0]
        _need(kv_len.dtype == torch.int32 and kv_len.shape == (n,) and kv_len.is_contiguous(),
              "kv_len must be int32 [n_seqs]")
        if cu_rows is None:
            _need(rows is None or rows == n, "without cu_rows there is one row for each sequence")
            rows = n
        else:
            _need(cu_rows.dtype == torch.int32 and cu_rows.shape == (n + 1,) and cu_rows.is_contiguous(),
                  "cu_rows must be int32 [n_seqs + 1]")
            _need(rows is not None, "cu_rows needs rows")
            _need(cu_rows.device == kv_len.device, "the batch's tensors are on several devices")
        _need(page_table.device == kv_len.device, "the batch's tensors are on several devices")
        self.page_table, self.kv_len, self.cu_rows, self.rows = page_table, kv_len, cu_rows, int(rows)
        self.device = kv_len.device
        max_len = page_table.shape[1] * 128 if max_len is None else int(max_len)
        self.struct = _a.batch_struct(page_table, kv_len, cu_rows, self.rows, max_len)
        if n <= 1:
            self.struct.page_table_stride = page_table.shape[1]      # (the stride of a single row says nothing)
        self.ref = ctypes.byref(self.struct)
        self._workspace = {}

    def workspace_bytes(self, cache, q_heads):
        key = (q_heads, cache.kv_heads, cache.head_dim, cache.page_size)
        if key not in self._workspace:
            self._workspace[key] = _a.nvfp4_kv_attention_workspace(cache.ref, self.ref, q_heads)
        return self._workspace[key]


def _gamma_ok(gamma, dim, name):
    if gamma is not None:
        _need(gamma.dtype == torch.bfloat16 and gamma.shape == (dim,) and gamma.is_contiguous(),
              "%s must be bf16 [head_dim]" % name)


def _positions_ok(positions, rows):
    _need(positions.dtype == torch.int32 and positions.shape == (rows,) and positions.is_contiguous(),
          "positions must be int32 [rows]")


def qk_norm_rope(q, k, positions=None, rope: Rope = None, q_gamma=None, k_gamma=None, eps=1e-6, q_out=None, k_out=None,
                 stream=None):
    """RMSNorm of each head of q and of k (either may be None; no norm without
    its gamma) and the rotation of its first elements by ``positions`` (int32
    [rows]), in one pass.  Returns (q, k); q_out and k_out may be q and k."""
    one = q if q is not None else k
    _need(one is not None, "q or k must be given")
    dim, rows = one.shape[-1], one.shape[0]
    inv_freq = rope.inv_freq if rope is not None else None
    for name, x, gamma in (("q", q, q_gamma), ("k", k, k_gamma)):
        if x is not None:
            _rows_ok(x, None, dim, name)
            _need(x.shape[0] == rows and x.device == one.device, "q and k differ in rows or device")
            _gamma_ok(gamma, dim, name + "_gamma")
    if inv_freq is not None:
        _need(positions is not None, "a rotation needs positions")
        _positions_ok(positions, rows)
    if q is not None:
        q_out = _like_rows(q, stream) if q_out is None else q_out
        _rows_ok(q_out, q.shape[1], dim, "q_out")
        _need(q_out.shape[0] == rows, "q_out has the wrong rows")
    if k is not None:
        k_out = _like_rows(k, stream) if k_out is None else k_out
        _rows_ok(k_out, k.shape[1], dim, "k_out")
        _need(k_out.shape[0] == rows, "k_out has the wrong rows")
    _run(one, _a.nvfp4_qk_norm_rope, q, q_gamma, q_out, k, k_gamma, k_out, eps, positions if inv_freq is not None else None,
         inv_freq, 0 if rope is None else rope.interleaved, stream)
    return (q_out if q is not None else None), (k_out if k is not None else None)


def kv_append(cache: KVCache, batch: Batch, k, v, k_gamma=None, eps=1e-6, rope: Rope = None, positions=None,
              static=False, stream=None):
    """Append a step's keys (normed and rotated on the way, each token by its
    number in its sequence unless ``positions`` are given) and values to the
    cache, with scales taken from the values, or the cache's own if ``static``."""
    _rows_ok(k, cache.kv_heads, cache.head_dim, "k")
    _rows_ok(v, cache.kv_heads, cache.head_dim, "v")
    _need(k.shape[0] == v.shape[0] == batch.rows, "k and v must have the batch's rows")
    _need(k.device == v.device == cache.device == batch.device, "tensors are on several devices")
    _gamma_ok(k_gamma, cache.head_dim, "k_gamma")
    if positions is not None:
        _positions_ok(positions, batch.rows)
    inv_freq = rope.inv_freq if rope is not None else None
    _run(k, _a.nvfp4_kv_append, cache.ref, batch.ref, k, v, k_gamma, eps, positions, inv_freq,
         0 if rope is None else rope.interleaved, _c.NVFP4_STATIC if static else _c.NVFP4_DYNAMIC, stream)


def attention(q, cache: KVCache, batch: Batch, scale=None, causal=True, window=0, out=None, return_lse=False,
              workspace=None, stream=None):
    """Attention of a step's queries over the cache, which holds the step's own
    tokens already.  ``scale``: 1 / sqrt(head_dim) unless given.  Returns y
    (bf16, q's shape), with the rows' log-sum-exp (float32 [rows, q_heads]) if
    ``return_lse``.  Rows behind the batch's last sequence are left as they are."""
    _rows_ok(q, None, cache.head_dim, "q")
    _need(q.shape[0] == batch.rows and q.shape[1] % cache.kv_heads == 0, "q has the wrong rows or heads")
    _need(q.device == cache.device == batch.device, "tensors are on several devices")
    y = _like_rows(q, stream) if out is None else out
    if out is not None:
        _rows_ok(y, q.shape[1], cache.head_dim, "out")
        _need(y.shape[0] == q.shape[0] and y.device == q.device, "out has the wrong rows or device")
    lse = None
    if return_lse:
        with _l._on(stream, q.device):
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    if workspace is None:
        nbytes = batch.workspace_bytes(cache, q.shape[1])
        workspace = _l._scratch(nbytes, q.device, stream) if nbytes else None
    scale = 1.0 / math.sqrt(cache.head_dim) if scale is None else scale
    _run(q, _a.nvfp4_kv_attention, cache.ref, batch.ref, q, y, lse, scale, 1 if causal else 0, window, workspace, stream)
    return (y, lse) if return_lse else y
