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
There is no backward pass: a tensor that requires a gradient is refused, unless
gradients are off (torch.no_grad(), torch.inference_mode()).
"""

import ctypes
import math

import torch

from . import linear as _l
from . import nvfp4_attention as _a


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# These checks run once a call and layer, in front of kernels of a few
# microseconds: no formatted text, no tensor property read twice.

_BF16 = torch.bfloat16
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)      # (the raw query: 0.1 us less)


def _no_gradient(name):
    if torch.is_grad_enabled():
        raise ValueError(name + " requires a gradient, and none passes through here")


def _rows(x, name):
    """(rows, heads, head_dim, row stride) of a bf16 [rows, heads, head_dim]
    tensor whose heads lie side by side (the stride of a single row says nothing)."""
    if x.dtype is not _BF16 or x.dim() != 3:
        raise ValueError(name + " must be a bf16 [rows, heads, head_dim] tensor")
    if x.requires_grad:
        _no_gradient(name)
    rows, heads, dim = x.shape
    ld, head, one = x.stride()
    if (one != 1 or (head != dim and heads > 1)) and rows * heads * dim > 0:
        raise ValueError(name + " must have its heads side by side")
    return rows, heads, dim, ld if rows > 1 else heads * dim


def _like_rows(x, stream):
    """A contiguous [rows, heads, head_dim] tensor from the stream that uses it.
    (empty_like closes the gaps between x's rows.)"""
    if stream is None:
        return torch.empty_like(x)
    with _l._on(stream, x.device):
        return torch.empty_like(x)


def _run(device, call, stream, *args):
    """``call(stream, *args)`` with that device current (kernels are launched on
    the current device, on its current stream); no context where it is already."""
    if device < 0:
        raise ValueError("tensors must be on the GPU, on one device")
    if device == _current_device():
        return call(stream, *args)
    with torch.cuda.device(device):
        return call(stream, *args)


class Rope:
    """The rotation of a head's first 2 * len(inv_freq) elements by the angles
    position * inv_freq[i] (float32, on the GPU): element i with element
    i + len(inv_freq), or 2 i with 2 i + 1 if ``interleaved``."""

    def __init__(self, inv_freq, interleaved=False):
        _need(inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.shape[0] % 8 == 0,
              "inv_freq must be a float32 vector of a multiple of 8 elements")
        _need(not inv_freq.requires_grad, "inv_freq takes no gradient here")
        self.inv_freq = inv_freq.contiguous()
        self.device = self.inv_freq.get_device()
        half = inv_freq.shape[0]
        self.pointer = (self.inv_freq.data_ptr() if half else None, half, 1 if interleaved else 0)


class KVCache:
    """A layer's paged cache over given buffers: k, v uint8 [num_pages,
    kv_heads, page_size * head_dim] in the order that nvfp4_attention.h states
    (any page stride that is a multiple of 16), k_scale, v_scale float32
    [num_pages, kv_heads] with one row stride.  (Strides of a single page say nothing.)"""

    def __init__(self, k, v, k_scale, v_scale, page_size):
        for name, t in (("k", k), ("v", v)):
            _need(t.dtype == torch.uint8 and t.dim() == 3 and t.shape == k.shape and t.shape[2] % page_size == 0,
                  "%s must be uint8 [num_pages, kv_heads, page_size * head_dim]" % name)
            _need(t.stride(2) == 1 and (t.shape[1] == 1 or t.stride(1) == t.shape[2]),
                  "the heads of a page of %s must be side by side" % name)
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _need(t.dtype == torch.float32 and t.shape == k.shape[:2]
                  and (t.stride(0) == k_scale.stride(0) or t.shape[0] == 1)
                  and (t.shape[1] == 1 or t.stride(1) == 1), "%s must be float32 [num_pages, kv_heads]" % name)
            _need(not t.requires_grad, "%s takes no gradient here" % name)
        _need(k.device == v.device == k_scale.device == v_scale.device, "the cache's buffers are on several devices")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.page_size, self.kv_heads, self.head_dim = page_size, k.shape[1], k.shape[2] // page_size
        self.device, self.index = k.device, k.get_device()
        self.softmax_scale = 1.0 / math.sqrt(self.head_dim)
        self.struct = _a.cache_struct(k, v, k_scale, v_scale, page_size)
        if k.shape[0] == 1:
            self.struct.k_page_stride = self.struct.v_page_stride = k.shape[1] * k.shape[2]
            self.struct.scale_page_stride = k.shape[1]
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
    ``kv_append(..., static=True)``): one number, or the keys' and the values'."""
    both = scale if isinstance(scale, (tuple, list)) else (scale, scale)
    _need(len(both) == 2, "scale must be a number or the keys' and the values'")
    codes = [torch.empty((num_pages, kv_heads, page_size * head_dim), dtype=torch.uint8, device=device)
             for _ in range(2)]
    scales = [torch.full((num_pages, kv_heads), 0.0 if s is None else float(s), dtype=torch.float32, device=device)
              for s in both]
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
        self.device, self.index = kv_len.device, kv_len.get_device()
        max_len = page_table.shape[1] * 128 if max_len is None else int(max_len)
        self.struct = _a.batch_struct(page_table, kv_len, cu_rows, self.rows, max_len)
        if n <= 1:
            self.struct.page_table_stride = page_table.shape[1]      # (the stride of a single row says nothing)
        self.ref = ctypes.byref(self.struct)
        self._workspace = {}

    def workspace_bytes(self, cache, q_heads):
        key = (q_heads, cache.kv_heads, cache.head_dim, cache.page_size)
        if key not in self._workspace:
            self._workspace[key] = _a.kv_attention_workspace(cache.ref, self.ref, q_heads)
        return self._workspace[key]


# Devices are compared by their indices (below 0: not a GPU).

def _gamma(gamma, dim, device, name):
    """Address of a bf16 [head_dim] vector, or None."""
    if gamma is None:
        return None
    if gamma.requires_grad:
        _no_gradient(name)
    if gamma.dtype is not _BF16 or gamma.dim() != 1 or gamma.numel() != dim or not gamma.is_contiguous():
        raise ValueError(name + " must be bf16 [head_dim]")
    if gamma.get_device() != device:
        raise ValueError(name + " is on another device")
    return gamma.data_ptr()


def _positions(positions, rows, device):
    if positions is None:
        return None
    if positions.dtype is not torch.int32 or positions.dim() != 1 or positions.numel() != rows \
            or not positions.is_contiguous():
        raise ValueError("positions must be int32 [rows]")
    if positions.get_device() != device:
        raise ValueError("positions are on another device")
    return positions.data_ptr()


def _rotation(rope, device):
    """(inv_freq's address, its elements, interleaved)."""
    if rope is None:
        return None, 0, 0
    if rope.device != device:
        raise ValueError("the rotation's inv_freq is on another device")
    return rope.pointer


_Q_NAMES, _K_NAMES = ("q", "q_gamma", "q_out"), ("k", "k_gamma", "k_out")


def _head_args(x, gamma, y, rows, dim, device, names, stream):
    """((x, stride, heads, gamma, y, stride), y) of the queries or the keys."""
    if x is None:
        return (None, 0, 0, None, None, 0), None
    n, heads, d, ld = _rows(x, names[0])
    if n != rows or d != dim or x.get_device() != device:
        raise ValueError("q and k differ in rows, head_dim or device")
    if y is None:
        y, ldy = _like_rows(x, stream), heads * d
    else:
        ny, hy, dy, ldy = _rows(y, names[2])
        if ny != n or hy != heads or dy != d or y.get_device() != device:
            raise ValueError(names[2] + " must have the shape and device of its input")
    return (x.data_ptr(), ld, heads, None if gamma is None else _gamma(gamma, d, device, names[1]), y.data_ptr(), ldy), y


def qk_norm_rope(q, k, positions=None, rope: Rope = None, q_gamma=None, k_gamma=None, eps=1e-6, q_out=None, k_out=None,
                 stream=None):
    """RMSNorm of each head of q and of k (either may be None; no norm without
    its gamma) and the rotation of its first elements by ``positions`` (int32
    [rows]), in one pass.  Returns (q, k); q_out and k_out may be q and k."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("q or k must be given")
    rows, dim, device = one.shape[0], one.shape[-1], one.get_device()
    q_args, q_out = _head_args(q, q_gamma, q_out, rows, dim, device, _Q_NAMES, stream)
    k_args, k_out = _head_args(k, k_gamma, k_out, rows, dim, device, _K_NAMES, stream)
    inv_freq, half, interleaved = _rotation(rope, device)
    if half and positions is None:
        raise ValueError("a rotation needs positions")
    _run(device, _a.qk_norm_rope, stream, *q_args, *k_args, rows, dim, eps,
         _positions(positions, rows, device) if half else None, inv_freq, 2 * half, interleaved)
    return q_out, k_out


def kv_append(cache: KVCache, batch: Batch, k, v, k_gamma=None, eps=1e-6, rope: Rope = None, positions=None,
              static=False, stream=None):
    """Append a step's keys (normed and rotated on the way, each token by its
    number in its sequence unless ``positions`` are given) and values to the
    cache, with scales taken from the values, or the cache's own if ``static``."""
    rows, heads, dim, ldk = _rows(k, "k")
    rows_v, heads_v, dim_v, ldv = _rows(v, "v")
    if rows != batch.rows or rows_v != rows:
        raise ValueError("k and v must have the batch's rows")
    if heads != cache.kv_heads or heads_v != heads or dim != cache.head_dim or dim_v != dim:
        raise ValueError("k and v must have the cache's heads and head_dim")
    device = k.get_device()
    if not device == v.get_device() == cache.index == batch.index:
        raise ValueError("tensors are on several devices")
    inv_freq, half, interleaved = _rotation(rope, device)
    _run(device, _a.kv_append, stream, cache.ref, batch.ref, k.data_ptr(), ldk, v.data_ptr(), ldv,
         _gamma(k_gamma, dim, device, "k_gamma"), eps, _positions(positions, rows, device), inv_freq, 2 * half, interleaved, 1 if static else 0)


def attention(q, cache: KVCache, batch: Batch, scale=None, causal=True, window=0, out=None, return_lse=False,
              workspace=None, stream=None):
    """Attention of a step's queries over the cache, which holds the step's own
    tokens already.  ``scale``: 1 / sqrt(head_dim) unless given.  Returns y
    (bf16, q's shape), with the rows' log-sum-exp (float32 [rows, q_heads]) if
    ``return_lse``.  Rows behind the batch's last sequence are left as they are."""
    rows, heads, dim, ldq = _rows(q, "q")
    if rows != batch.rows or dim != cache.head_dim or heads == 0 or heads % cache.kv_heads:
        raise ValueError("q has the wrong rows, heads or head_dim")
    device = q.get_device()
    if not device == cache.index == batch.index:
        raise ValueError("tensors are on several devices")
    if out is None:
        y, ldy = _like_rows(q, stream), heads * dim
    else:
        y = out
        rows_y, heads_y, dim_y, ldy = _rows(y, "out")
        if (rows_y, heads_y, dim_y) != (rows, heads, dim) or y.get_device() != device:
            raise ValueError("out must have q's shape and device")
    lse = None
    if return_lse:
        with _l._on(stream, q.device):
            lse = torch.empty((rows, heads), dtype=torch.float32, device=q.device)
    if workspace is None:
        nbytes = batch.workspace_bytes(cache, heads)
        workspace = _l._scratch(nbytes, q.device, stream) if nbytes else None
    else:
        if workspace.get_device() != device or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous, on q's device")
        nbytes = workspace.numel() * workspace.element_size()
    _run(device, _a.kv_attention, stream, cache.ref, batch.ref, q.data_ptr(), ldq, heads, y.data_ptr(), ldy,
         None if lse is None else lse.data_ptr(), cache.softmax_scale if scale is None else scale, 1 if causal else 0,
         window, None if workspace is None else workspace.data_ptr(), nbytes)
    return (y, lse) if return_lse else y


def attention_kernels(q_heads, cache: KVCache, batch: Batch, window=0):
    """Names of the kernels that attention() launches for a step."""
    return [name for name in (_a.kv_attention_kernel(cache.ref, batch.ref, q_heads, window, part) for part in (0, 1))
            if name is not None]
