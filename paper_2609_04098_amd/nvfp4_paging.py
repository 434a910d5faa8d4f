"""ctypes binding of the paging entry points of libnvfp4.so
(include/nvfp4_paging.h): argument marshalling only.
"""

import ctypes

from . import nvfp4 as _c
from .nvfp4_attention import _batch, _cache, _f, _handle, _i64, _int, _sz, _vp


class RequestsStruct(ctypes.Structure):
    _fields_ = [("page_table", _vp), ("kv_len", _vp), ("free_pages", _vp), ("free_count", _vp),
                ("page_table_stride", _i64), ("max_pages", _i64), ("n_seqs", _i64), ("num_pages", _i64),
                ("page_size", _i64)]


class SharedPrefixStruct(ctypes.Structure):
    _fields_ = [("cu_seqs", _vp), ("prefix", _vp), ("n_groups", _i64), ("max_prefix", _i64), ("max_own", _i64)]


class BoundsStruct(ctypes.Structure):
    _fields_ = [("codes", _vp), ("step", _vp), ("page_stride", _i64), ("step_stride", _i64)]


_requests, _shared = ctypes.POINTER(RequestsStruct), ctypes.POINTER(SharedPrefixStruct)
_bounds = ctypes.POINTER(BoundsStruct)

# name -> (restype, argtypes), in the order of include/nvfp4_paging.h
SIGNATURES = {
    "nvfp4_step_tables_workspace": (_sz, [_i64]),
    "nvfp4_step_tables": (_int, [_requests, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp]),
    "nvfp4_kv_attention_shared_workspace": (_sz, [_cache, _batch, _shared, _i64]),
    "nvfp4_kv_attention_shared": (_int, [_cache, _batch, _shared, _vp, _i64, _i64, _vp, _i64, _vp, _f, _int, _vp, _sz,
                                         _vp]),
    "nvfp4_kv_attention_shared_kernel": (ctypes.c_char_p, [_cache, _batch, _shared, _i64, _int]),
    "nvfp4_kv_page_bounds": (_int, [_cache, _batch, _bounds, _vp]),
    "nvfp4_kv_select_pages_workspace": (_sz, [_cache, _batch]),
    "nvfp4_kv_select_pages": (_int, [_cache, _batch, _bounds, _vp, _i64, _i64, _i64, _i64, _i64, _int, _vp, _vp, _vp, _vp,
                                     _sz, _vp]),
    "nvfp4_kv_attention_selected_workspace": (_sz, [_cache, _i64, _i64, _i64]),
    "nvfp4_kv_attention_selected": (_int, [_cache, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _f, _vp, _sz,
                                           _vp]),
}

_lib = None


def lib():
    """The loaded library with the paging entry points declared."""
    global _lib
    if _lib is None:
        l = _c.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def requests_struct(page_table, kv_len, free_pages, free_count, page_size):
    """page_table int32 [n_seqs, max_pages]; kv_len int32 [n_seqs]; free_pages
    int32 [num_pages]; free_count int32 [1]."""
    return RequestsStruct(page_table.data_ptr(), kv_len.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
                          page_table.stride(0), page_table.shape[1], kv_len.shape[0], free_pages.shape[0], page_size)


def shared_struct(cu_seqs, prefix, max_prefix, max_own):
    """cu_seqs int32 [n_groups + 1]; prefix int32 [n_groups]."""
    return SharedPrefixStruct(cu_seqs.data_ptr(), prefix.data_ptr(), prefix.shape[0], max_prefix, max_own)


def bounds_struct(codes, step):
    """codes int8 [num_pages, kv_heads, 2, head_dim]; step float32 [num_pages, kv_heads]."""
    return BoundsStruct(codes.data_ptr(), step.data_ptr(), codes.stride(0), step.stride(0))


def step_tables_workspace(n_seqs):
    return lib().nvfp4_step_tables_workspace(n_seqs)


def step_tables(stream, *args):
    """nvfp4_step_tables: its arguments in order, addresses as integers (or None), the
    structure by reference, after the stream: a torch stream, a handle or None (the
    current one)."""
    status = (_lib or lib()).nvfp4_step_tables(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_step_tables")


def kv_attention_shared_workspace(cache, batch, shared, q_heads):
    return lib().nvfp4_kv_attention_shared_workspace(cache, batch, shared, q_heads)


def kv_attention_shared(stream, *args):
    """nvfp4_kv_attention_shared, its arguments as above."""
    status = (_lib or lib()).nvfp4_kv_attention_shared(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_attention_shared")


def kv_attention_shared_kernel(cache, batch, shared, q_heads, part=0):
    """Name of launch `part` of nvfp4_kv_attention_shared for these sizes, or None."""
    r = lib().nvfp4_kv_attention_shared_kernel(cache, batch, shared, q_heads, part)
    return None if r is None else r.decode()


def kv_page_bounds(stream, *args):
    """nvfp4_kv_page_bounds, its arguments as above."""
    status = (_lib or lib()).nvfp4_kv_page_bounds(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_page_bounds")


def kv_select_pages_workspace(cache, batch):
    return lib().nvfp4_kv_select_pages_workspace(cache, batch)


def kv_select_pages(stream, *args):
    """nvfp4_kv_select_pages, its arguments as above."""
    status = (_lib or lib()).nvfp4_kv_select_pages(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_select_pages")


def kv_attention_selected_workspace(cache, rows, q_heads, count):
    return lib().nvfp4_kv_attention_selected_workspace(cache, rows, q_heads, count)


def kv_attention_selected(stream, *args):
    """nvfp4_kv_attention_selected, its arguments as above."""
    status = (_lib or lib()).nvfp4_kv_attention_selected(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_attention_selected")
