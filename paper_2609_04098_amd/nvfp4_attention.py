"""ctypes binding of the attention entry points of libnvfp4.so
(include/nvfp4_attention.h): argument marshalling only.
"""

import ctypes

from . import nvfp4 as _c

_i64, _vp, _sz, _int, _f = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float


class KvCacheStruct(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("num_pages", _i64), ("page_size", _i64),
                ("kv_heads", _i64), ("head_dim", _i64), ("k_page_stride", _i64), ("v_page_stride", _i64),
                ("scale_page_stride", _i64)]


class KvBatchStruct(ctypes.Structure):
    _fields_ = [("page_table", _vp), ("kv_len", _vp), ("cu_rows", _vp), ("page_table_stride", _i64),
                ("max_pages", _i64), ("n_seqs", _i64), ("rows", _i64), ("max_kv_len", _i64)]


_cache, _batch = ctypes.POINTER(KvCacheStruct), ctypes.POINTER(KvBatchStruct)

# name -> (restype, argtypes), in the order of include/nvfp4_attention.h
SIGNATURES = {
    "nvfp4_qk_norm_rope": (_int, [_vp, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _f,
                                  _vp, _vp, _i64, _int, _vp]),
    "nvfp4_kv_append": (_int, [_cache, _batch, _vp, _i64, _vp, _i64, _vp, _f, _vp, _vp, _i64, _int, _int, _vp]),
    "nvfp4_kv_attention_workspace": (_sz, [_cache, _batch, _i64]),
    "nvfp4_kv_attention": (_int, [_cache, _batch, _vp, _i64, _i64, _vp, _i64, _vp, _f, _int, _i64, _vp, _sz, _vp]),
    "nvfp4_kv_attention_kernel": (ctypes.c_char_p, [_cache, _batch, _i64, _i64, _int]),
}

_lib = None


def lib():
    """The loaded library with the attention entry points declared."""
    global _lib
    if _lib is None:
        l = _c.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def _at(t):
    return None if t is None else t.data_ptr()


def cache_struct(k, v, k_scale, v_scale, page_size):
    """k, v uint8 [num_pages, kv_heads, page_size * head_dim]; k_scale, v_scale
    float32 [num_pages, kv_heads]."""
    return KvCacheStruct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k.shape[0], page_size,
                         k.shape[1], k.shape[2] // page_size, k.stride(0), v.stride(0), k_scale.stride(0))


def batch_struct(page_table, kv_len, cu_rows, rows, max_kv_len):
    """page_table int32 [n_seqs, max_pages]; kv_len int32 [n_seqs]; cu_rows
    int32 [n_seqs + 1] or None."""
    return KvBatchStruct(page_table.data_ptr(), kv_len.data_ptr(), _at(cu_rows), page_table.stride(0),
                         page_table.shape[1], kv_len.shape[0], rows, max_kv_len)


def _handle(stream):
    """Handle of a torch stream, a handle itself, or of the current stream (None)."""
    return _c._current_stream() if stream is None else getattr(stream, "cuda_stream", stream)


def qk_norm_rope(stream, *args):
    """nvfp4_qk_norm_rope: its arguments in order, addresses as integers (or
    None), after the stream: a torch stream, a handle or None (the current one)."""
    status = (_lib or lib()).nvfp4_qk_norm_rope(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_qk_norm_rope")


def kv_append(stream, *args):
    """nvfp4_kv_append, its arguments as above, the structures by reference."""
    status = (_lib or lib()).nvfp4_kv_append(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_append")


def kv_attention_workspace(cache, batch, q_heads):
    return lib().nvfp4_kv_attention_workspace(cache, batch, q_heads)


def kv_attention(stream, *args):
    """nvfp4_kv_attention, its arguments as above."""
    status = (_lib or lib()).nvfp4_kv_attention(*args, _handle(stream))
    if status:
        _c._check(status, "nvfp4_kv_attention")


def kv_attention_kernel(cache, batch, q_heads, window=0, part=0):
    """Name of launch `part` of nvfp4_kv_attention for these sizes, or None."""
    r = lib().nvfp4_kv_attention_kernel(cache, batch, q_heads, window, part)
    return None if r is None else r.decode()
