"""Serving over the paged 8-bit cache of ``attention``, on top of the C ABI
(include/nvfp4_paging.h): argument checks, buffers and call order only.

    requests = alloc_requests(n_seqs, max_pages, num_pages, page_size, device)   # once: lengths, pages, the pool
    step = step_tables(requests, new_rows, rows, drop)    # per step: page tables, row offsets, positions, slots
    attention.kv_append(cache, step.batch, k, v, ...)
    shared = SharedPrefix(cu_seqs, prefix)                # while the groups stay the same
    y = shared_attention(q, cache, step.batch, shared)    # attention(q, cache, step.batch), prefixes read once

    bounds = alloc_page_bounds(cache)                     # per layer
    page_bounds(cache, step.batch, bounds)                # behind each append
    pages = select_pages(q, cache, step.batch, bounds, count)   # for each row and key head
    y = selected_attention(q, cache, pages)

Lengths stay on the GPU: nothing here waits for it, and every call may be captured
into a graph.  There is no backward pass, as in ``attention``.
"""

import ctypes

import torch

from . import attention as _at
from . import linear as _l
from . import nvfp4_paging as _p
from .attention import Batch, KVCache, _like_rows, _need, _rows, _run

_I32 = torch.int32


def _vector(t, n, device, name):
    """Address of an int32 [n] vector on the device, or None."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(name + " must be int32, one number for each sequence")
    if t.get_device() != device:
        raise ValueError(name + " is on another device")
    return t.data_ptr()


class Requests:
    """The sequences of a serving loop over given buffers, all on one GPU:
    page_table int32 [n_seqs, max_pages], kv_len int32 [n_seqs] (tokens held),
    free_pages int32 [num_pages] of which the first free_count [1] are the free pages'
    numbers (the last of them the next to be taken)."""

    def __init__(self, page_table, kv_len, free_pages, free_count, page_size):
        _need(page_size in (16, 32, 64, 128), "page_size must be 16, 32, 64 or 128")
        _need(page_table.dtype == _I32 and page_table.dim() == 2
              and (page_table.shape[1] <= 1 or page_table.stride(1) == 1), "page_table must be int32 [n_seqs, max_pages]")
        _need(kv_len.dtype == _I32 and kv_len.shape == page_table.shape[:1] and kv_len.is_contiguous(),
              "kv_len must be int32 [n_seqs]")
        _need(free_pages.dtype == _I32 and free_pages.dim() == 1 and free_pages.shape[0] > 0
              and free_pages.is_contiguous(), "free_pages must be int32 [num_pages]")
        _need(free_count.dtype == _I32 and free_count.shape == (1,), "free_count must be int32 [1]")
        _need(page_table.device == kv_len.device == free_pages.device == free_count.device,
              "the requests' tensors are on several devices")
        _need(page_table.shape[0] <= 1 or page_table.stride(0) >= page_table.shape[1],
              "rows of page_table must not overlap")
        self.page_table, self.kv_len, self.free_pages, self.free_count = page_table, kv_len, free_pages, free_count
        self.page_size, self.n_seqs = page_size, kv_len.shape[0]
        self.device, self.index = kv_len.device, kv_len.get_device()
        self.struct = _p.requests_struct(page_table, kv_len, free_pages, free_count, page_size)
        if self.n_seqs <= 1:
            self.struct.page_table_stride = page_table.shape[1]      # (the stride of a single row says nothing)
        self.ref = ctypes.byref(self.struct)


def alloc_requests(n_seqs, max_pages, num_pages, page_size, device):
    """Sequences without tokens, all pages free (page 0 is the first to be taken)."""
    return Requests(torch.zeros((n_seqs, max_pages), dtype=_I32, device=device),
                    torch.zeros(n_seqs, dtype=_I32, device=device),
                    torch.arange(num_pages - 1, -1, -1, dtype=_I32, device=device),
                    torch.full((1,), num_pages, dtype=_I32, device=device), page_size)


class Step:
    """A step's tables: ``batch`` (what kv_append and the attentions take, over the
    requests' page_table and kv_len), ``positions`` int32 [rows], ``slots`` int64 [rows]
    (page * page_size + slot).  ``batch.cu_rows`` says which rows each sequence got."""

    def __init__(self, requests, rows, max_len=None):
        n, device = requests.n_seqs, requests.device
        self.requests, self.rows, self.max_len = requests, int(rows), max_len
        cu_rows = torch.empty(n + 1, dtype=_I32, device=device)
        self.batch = _at.Batch(requests.page_table, requests.kv_len, cu_rows, rows=self.rows, max_len=max_len)
        self.positions = torch.empty(self.rows, dtype=_I32, device=device)
        self.slots = torch.empty(self.rows, dtype=torch.int64, device=device)
        nbytes = _p.step_tables_workspace(n)
        self._workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self._args = (cu_rows.data_ptr(), self.positions.data_ptr(), self.slots.data_ptr(), self.rows,
                      self._workspace.data_ptr(), nbytes)


def step_tables(requests: Requests, new_rows, rows, drop=None, kept=None, max_len=None, out: Step = None, stream=None):
    """Takes ``drop`` tokens (int32 [n_seqs], or None) off the sequences' ends and adds
    ``new_rows`` (int32 [n_seqs]) to them: pages go back to the pool and come from it,
    page_table, kv_len and the pool change in place.  ``rows``: rows of the step's
    tensors.  ``kept``: tokens in front of each sequence whose pages never go back (a
    shared prefix).  From the first sequence for which pages or rows are missing on,
    none gets rows; one that its row of page_table cannot hold gets none either.
    ``out``: a Step of an earlier call, whose buffers are written again (always in a
    captured loop); ``max_len`` as for Batch."""
    device = requests.index
    if out is None:
        with _l._on(stream, requests.device):
            out = Step(requests, rows, max_len)
    elif out.requests is not requests or out.rows != rows or out.max_len != max_len:
        raise ValueError("out is a step of other requests, rows or max_len")
    n = requests.n_seqs
    if new_rows is None:
        raise ValueError("new_rows must be given")
    _run(device, _p.step_tables, stream, requests.ref, _vector(new_rows, n, device, "new_rows"),
         _vector(drop, n, device, "drop"), _vector(kept, n, device, "kept"), *out._args)
    return out


class SharedPrefix:
    """Groups of a batch's sequences that share a prefix, on the GPU: sequences
    [cu_seqs[g], cu_seqs[g + 1]) begin with the same ``prefix[g]`` tokens in the same
    pages (int32 [n_groups + 1] and [n_groups]).  ``max_len``, ``max_own``: the longest
    prefix and the most tokens of a sequence behind it, as far as the host knows (else
    what the page table can hold): work is divided by them."""

    def __init__(self, cu_seqs, prefix, max_len=None, max_own=None):
        _need(prefix.dtype == _I32 and prefix.dim() == 1 and prefix.is_contiguous(), "prefix must be int32 [n_groups]")
        _need(cu_seqs.dtype == _I32 and cu_seqs.shape == (prefix.shape[0] + 1,) and cu_seqs.is_contiguous(),
              "cu_seqs must be int32 [n_groups + 1]")
        _need(cu_seqs.device == prefix.device, "the groups' tensors are on several devices")
        most = (1 << 31) - 1
        self.cu_seqs, self.prefix, self.index = cu_seqs, prefix, prefix.get_device()
        self.struct = _p.shared_struct(cu_seqs, prefix, most if max_len is None else int(max_len),
                                       most if max_own is None else int(max_own))
        self.ref = ctypes.byref(self.struct)
        self._workspace = {}

    def workspace_bytes(self, cache, batch, q_heads):
        b = batch.struct
        key = (q_heads, cache.kv_heads, cache.head_dim, cache.page_size, b.rows, b.n_seqs, b.max_pages, b.max_kv_len,
               b.cu_rows is None)
        if key not in self._workspace:
            self._workspace[key] = _p.kv_attention_shared_workspace(cache.ref, batch.ref, self.ref, q_heads)
        return self._workspace[key]


def _queries(q, cache, rows, out, stream):
    """(rows, heads, q's row stride, y, y's row stride) of an attention's queries and output."""
    n, heads, dim, ldq = _rows(q, "q")
    if n != rows or dim != cache.head_dim or heads == 0 or heads % cache.kv_heads:
        raise ValueError("q has the wrong rows, heads or head_dim")
    if q.get_device() != cache.index:
        raise ValueError("tensors are on several devices")
    if out is None:
        return n, heads, ldq, _like_rows(q, stream), heads * dim
    rows_y, heads_y, dim_y, ldy = _rows(out, "out")
    if (rows_y, heads_y, dim_y) != (n, heads, dim) or out.get_device() != cache.index:
        raise ValueError("out must have q's shape and device")
    return n, heads, ldq, out, ldy


def _room(workspace, nbytes, device, index, stream):
    """(workspace, its bytes): the given one, or one of nbytes from the stream that uses it."""
    if workspace is None:
        return (_l._scratch(nbytes, device, stream), nbytes) if nbytes else (None, 0)
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous, on q's device")
    return workspace, workspace.numel() * workspace.element_size()


def _lse(rows, heads, device, stream):
    if stream is None:
        return torch.empty((rows, heads), dtype=torch.float32, device=device)
    with _l._on(stream, device):
        return torch.empty((rows, heads), dtype=torch.float32, device=device)


def shared_attention(q, cache: KVCache, batch: Batch, shared: SharedPrefix, scale=None, causal=True, out=None,
                     return_lse=False, workspace=None, stream=None):
    """``attention(q, cache, batch)`` of sequences that share prefixes, which are read
    once for each group.  A sequence whose rows do not all lie behind the prefix is
    computed from its own pages alone.  Steps with prefixes below 1536 tokens, or with 64
    and more rows of a key head's query heads for an average sequence, take attention()'s
    kernels.  Arguments and results as for attention()."""
    rows, heads, ldq, y, ldy = _queries(q, cache, batch.rows, out, stream)
    if not cache.index == batch.index == shared.index:
        raise ValueError("tensors are on several devices")
    if shared.struct.n_groups > batch.struct.n_seqs:
        raise ValueError("there are more groups than sequences")
    lse = _lse(rows, heads, cache.device, stream) if return_lse else None
    workspace, nbytes = _room(workspace, 0 if workspace is not None else shared.workspace_bytes(cache, batch, heads),
                              cache.device, cache.index, stream)
    _run(cache.index, _p.kv_attention_shared, stream, cache.ref, batch.ref, shared.ref, q.data_ptr(), ldq, heads,
         y.data_ptr(), ldy, None if lse is None else lse.data_ptr(), cache.softmax_scale if scale is None else scale,
         1 if causal else 0, None if workspace is None else workspace.data_ptr(), nbytes)
    return (y, lse) if return_lse else y


def shared_attention_kernels(q_heads, cache: KVCache, batch: Batch, shared: SharedPrefix):
    """Names of the kernels that shared_attention() launches for a step."""
    return [name for name in (_p.kv_attention_shared_kernel(cache.ref, batch.ref, shared.ref, q_heads, part) for part in (0, 1))
            if name is not None]


class PageBounds:
    """Bounds of the keys of a cache's full pages over given buffers: codes int8
    [num_pages, kv_heads, 2, head_dim] (largest, smallest; any page stride that is a
    multiple of 16), step float32 [num_pages, kv_heads] (nvfp4_paging.h)."""

    def __init__(self, codes, step):
        _need(codes.dtype == torch.int8 and codes.dim() == 4 and codes.shape[2] == 2 and codes[:1].is_contiguous()
              and (codes.shape[0] <= 1 or codes.stride(0) >= codes[0].numel()),
              "codes must be int8 [num_pages, kv_heads, 2, head_dim]")
        _need(step.dtype == torch.float32 and step.shape == codes.shape[:2] and (step.shape[1] == 1 or step.stride(1) == 1)
              and (step.shape[0] <= 1 or step.stride(0) >= step.shape[1]), "step must be float32 [num_pages, kv_heads]")
        _need(not step.requires_grad, "step takes no gradient here")
        _need(codes.device == step.device, "the bounds' buffers are on several devices")
        self.codes, self.step, self.index = codes, step, codes.get_device()
        self.shape = (codes.shape[0], codes.shape[1], codes.shape[3])
        self.struct = _p.bounds_struct(codes, step)
        if codes.shape[0] == 1:      # (strides of a single page say nothing)
            self.struct.page_stride, self.struct.step_stride = codes[0].numel(), codes.shape[1]
        self.ref = ctypes.byref(self.struct)


def alloc_page_bounds(cache: KVCache):
    """Bounds of an empty cache's pages."""
    n, h = cache.k_scale.shape
    return PageBounds(torch.zeros((n, h, 2, cache.head_dim), dtype=torch.int8, device=cache.device),
                      torch.zeros((n, h), dtype=torch.float32, device=cache.device))


def _of_cache(bounds, cache, batch):
    if bounds.shape != (cache.struct.num_pages, cache.kv_heads, cache.head_dim):
        raise ValueError("the bounds are of another cache")
    if not cache.index == batch.index == bounds.index:
        raise ValueError("tensors are on several devices")


def page_bounds(cache: KVCache, batch: Batch, bounds: PageBounds, stream=None):
    """The bounds of the pages that a step's appended rows completed."""
    _of_cache(bounds, cache, batch)
    _run(cache.index, _p.kv_page_bounds, stream, cache.ref, batch.ref, bounds.ref)


# Bytes of scores that a choice may keep for as long as it lives.  (An allocation of their
# own takes the host 1.3 us.)
_FEW_SCORES = 1 << 20


class Selection:
    """The pages chosen for each row and key head: ``index`` int32 [rows, kv_heads, count]
    (numbers in the row's sequence, ascending, -1 behind them), ``pages`` (the same of the
    pages themselves) and ``tokens`` int32 [rows] (what the row sees of them; -1: a row
    behind the last sequence)."""

    def __init__(self, index, pages, tokens):
        for name, t in (("index", index), ("pages", pages)):
            _need(t.dtype == _I32 and t.dim() == 3 and t.shape == index.shape and t.is_contiguous(),
                  name + " must be int32 [rows, kv_heads, count]")
        _need(tokens.dtype == _I32 and tokens.shape == index.shape[:1] and tokens.is_contiguous(), "tokens must be int32 [rows]")
        _need(index.device == pages.device == tokens.device, "the selection's tensors are on several devices")
        self.index, self.pages, self.tokens, self.device_index = index, pages, tokens, index.get_device()
        self.shape = tuple(index.shape)
        self.pointers = (index.data_ptr(), pages.data_ptr(), tokens.data_ptr())

    @classmethod
    def _new(cls, rows, kv_heads, count, more, device, stream):
        """A new one with ``more`` bytes (a multiple of 16) of workspace, and the address of that."""
        self = cls.__new__(cls)
        n, front = rows * kv_heads * count, more // 4
        if stream is None:
            data = torch.empty(front + 2 * n + rows, dtype=_I32, device=device)
        else:
            with _l._on(stream, device):
                data = torch.empty(front + 2 * n + rows, dtype=_I32, device=device)
        self.shape, self.device_index = (rows, kv_heads, count), data.get_device()
        first = data.data_ptr()
        at = first + more
        self.pointers = (at, at + 4 * n, at + 8 * n)
        self._data, self._front, self._n = data, front, n
        return self, first

    def __getattr__(self, name):      # (tensors over one allocation, made where they are asked for)
        if name not in ("index", "pages", "tokens") or "_data" not in self.__dict__:
            raise AttributeError(name)
        n, at = self._n, self._front
        if name == "tokens":
            t = self._data[at + 2 * n:]
        else:
            t = (self._data[at:at + n] if name == "index" else self._data[at + n:at + 2 * n]).view(self.shape)
        self.__dict__[name] = t
        return t


def select_pages(q, cache: KVCache, batch: Batch, bounds: PageBounds, count, first=1, recent=1, causal=True,
                 out: Selection = None, workspace=None, stream=None) -> Selection:
    """Up to ``count`` pages for each of a step's rows and key heads: the ``first`` ones of
    its sequence, the ``recent`` ones of those that it sees, and between them those whose
    keys' bounds allow the largest products with a query of the key head (for a positive
    softmax scale; one with an infinity or a NaN among its elements has no say); all, where
    there are no more."""
    rows, heads, dim, ldq = _rows(q, "q")
    if rows != batch.rows or dim != cache.head_dim or heads == 0 or heads % cache.kv_heads:
        raise ValueError("q has the wrong rows, heads or head_dim")
    _of_cache(bounds, cache, batch)
    if q.get_device() != cache.index:
        raise ValueError("tensors are on several devices")
    count, first, recent = int(count), int(first), int(recent)
    if count < 1 or first < 0 or recent < 1 or first + recent > count:
        raise ValueError("first and recent pages must be among the count, with at least one recent page")
    if out is not None:
        if out.shape != (rows, cache.kv_heads, count):
            raise ValueError("out must be a selection of these rows, key heads and count")
        if out.device_index != cache.index:
            raise ValueError("out is on another device")
    nbytes, at, more = 0, None, 0
    if workspace is None:
        key = ("select", cache.kv_heads, cache.head_dim, cache.page_size)
        nbytes = batch._workspace.get(key)
        if nbytes is None:
            nbytes = batch._workspace[key] = (_p.kv_select_pages_workspace(cache.ref, batch.ref) + 15) & ~15
    if out is None:      # (the scores are this call's own; few are left in the choice's allocation)
        more = nbytes if nbytes <= _FEW_SCORES else 0
        out, at = Selection._new(rows, cache.kv_heads, count, more, cache.device, stream)
    if workspace is not None or nbytes > more:
        workspace, nbytes = _room(workspace, nbytes, cache.device, cache.index, stream)
        at = workspace.data_ptr()
    index, pages, tokens = out.pointers
    _run(cache.index, _p.kv_select_pages, stream, cache.ref, batch.ref, bounds.ref, q.data_ptr(), ldq, heads, count, first,
         recent, 1 if causal else 0, index, pages, tokens, at, nbytes)
    return out


def selected_attention(q, cache: KVCache, selection: Selection, scale=None, out=None, return_lse=False, workspace=None,
                       stream=None):
    """Attention of each row over the pages chosen for it.  Returns y (bf16, q's shape),
    with the log-sum-exp over those tokens if ``return_lse``."""
    n, kv_heads, count = selection.shape
    rows, heads, ldq, y, ldy = _queries(q, cache, n, out, stream)
    if kv_heads != cache.kv_heads:
        raise ValueError("the selection is of other key heads")
    if selection.device_index != cache.index:
        raise ValueError("tensors are on several devices")
    lse = _lse(rows, heads, cache.device, stream) if return_lse else None
    if workspace is None:
        key = (rows, count, heads)
        nbytes = cache.selected_workspace.get(key)
        if nbytes is None:
            nbytes = cache.selected_workspace[key] = _p.kv_attention_selected_workspace(cache.ref, rows, heads, count)
    else:
        nbytes = 0
    workspace, nbytes = _room(workspace, nbytes, cache.device, cache.index, stream)
    _, pages, tokens = selection.pointers
    _run(cache.index, _p.kv_attention_selected, stream, cache.ref, q.data_ptr(), ldq, heads, rows, count, pages, tokens,
         y.data_ptr(), ldy, None if lse is None else lse.data_ptr(), cache.softmax_scale if scale is None else scale,
         None if workspace is None else workspace.data_ptr(), nbytes)
    return (y, lse) if return_lse else y
