"""ctypes binding of the token operators of libuf.so (include/uft.h): argument marshalling only."""

import array
import ctypes

from . import _lib as L

UFT_MAX_TREE = 64


class uft_desc(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_seqs", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class uft_info(ctypes.Structure):
    _fields_ = [("free_pages", ctypes.c_int32), ("step_seqs", ctypes.c_int32), ("step_tokens", ctypes.c_int32),
                ("step_longest", ctypes.c_int32)]


class uft_stride(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class uft_attn_desc(ctypes.Structure):
    _fields_ = [("q_heads", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("n_cu", ctypes.c_int32), ("scale", ctypes.c_float), ("q", uft_stride)]


class uft_window_desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("window", ctypes.c_int32),
                ("sinks", ctypes.c_int32), ("scale", ctypes.c_float), ("q", uft_stride), ("k", uft_stride),
                ("v", uft_stride)]


_P, _I, _Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_IP, _ZP = ctypes.POINTER(_I), ctypes.POINTER(_Z)
_SIGNATURES = {
    "uft_pool_bytes": [ctypes.POINTER(uft_desc), _ZP],
    "uft_table_bytes": [ctypes.POINTER(uft_desc), _ZP],
    "uft_create": [ctypes.POINTER(uft_desc), _P, _Z, _P, _Z, ctypes.POINTER(_P)],
    "uft_destroy": [_P],
    "uft_extend": [_P, _I, _P, _P, _P],
    "uft_write": [_P, _I, _P, ctypes.POINTER(uft_stride), _P, ctypes.POINTER(uft_stride), _P],
    "uft_fork": [_P, _I, _P, _P, _P],
    "uft_copy": [_P, _I, _P, _P, _P],
    "uft_keep": [_P, _I, _P, _P, _P, _P, _P],
    "uft_trim": [_P, _I, _P, _I, _I, _P],
    "uft_free": [_P, _I, _P],
    "uft_pack": [_P, _IP, _P],
    "uft_get_info": [_P, ctypes.POINTER(uft_info)],
    "uft_seq_tokens": [_P, _I, _IP],
    "uft_seq_pages": [_P, _I, _IP, _I, _IP],
    "uft_attn_work_bytes": [_P, ctypes.POINTER(uft_attn_desc), _ZP],
    "uft_attn": [_P, _I, ctypes.POINTER(uft_attn_desc), _P, _P, _P, _P, _P, _Z, _P],
    "uft_window_fwd": [ctypes.POINTER(uft_window_desc), _P, _P, _P, _P, _P, _P, _P],
    "uft_window_bwd_work_bytes": [ctypes.POINTER(uft_window_desc), _ZP],
    "uft_window_bwd": [ctypes.POINTER(uft_window_desc)] + [_P] * 11 + [_Z, _P],
}

_lib = None


def load():
    """libuf.so with the signatures of the token operators."""
    global _lib
    if _lib is None:
        lib = L.load()
        for name, args in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = lib
    return _lib


def ints(values):
    """Host integers as the library reads them, an array of int32 (which the caller holds during the call)."""
    if isinstance(values, array.array) and values.typecode == "i":
        return values
    if hasattr(values, "data_ptr") or isinstance(values, (bytes, bytearray)):   # (an array would take those as its memory)
        raise TypeError(f"sequences, counts and starts are host integers, not {type(values).__name__}")
    return array.array("i", values)


def _at(ints):
    return ints.buffer_info()[0]


def _same(a, b, names):
    if len(a) != len(b):
        raise ValueError(f"{names} must have one entry for each sequence")


def _ref(x):
    return ctypes.byref(x)


def uft_pool_bytes(desc) -> int:
    out = _Z()
    L._check(load().uft_pool_bytes(_ref(desc), _ref(out)))
    return out.value


def uft_table_bytes(desc) -> int:
    out = _Z()
    L._check(load().uft_table_bytes(_ref(desc), _ref(out)))
    return out.value


def uft_create(desc, pool, table, pool_bytes=None, table_bytes=None):
    """pool, table: device tensors (or None under UF_F_DRYRUN). Returns the opaque handle."""
    h = _P()
    sizes = [n if n is not None else (0 if t is None else t.numel() * t.element_size())
             for t, n in ((pool, pool_bytes), (table, table_bytes))]
    L._check(load().uft_create(_ref(desc), L._ptr(pool), sizes[0], L._ptr(table), sizes[1], _ref(h)))
    return h


def uft_destroy(handle) -> None:
    L._check(load().uft_destroy(handle))


def uft_extend(handle, seqs, counts, stream=None) -> None:
    s, c = ints(seqs), ints(counts)
    _same(s, c, "seqs and counts")
    L._check(load().uft_extend(handle, len(s), _at(s), _at(c), stream))


def uft_write(handle, layer, k, k_stride, v, v_stride, stream=None) -> None:
    L._check(load().uft_write(handle, layer, L._ptr(k), _ref(k_stride), L._ptr(v), _ref(v_stride), stream))


def uft_fork(handle, src, dst, stream=None) -> None:
    s, d = ints(src), ints(dst)
    _same(s, d, "src and dst")
    L._check(load().uft_fork(handle, len(s), _at(s), _at(d), stream))


def uft_copy(handle, src, dst, stream=None) -> None:
    s, d = ints(src), ints(dst)
    _same(s, d, "src and dst")
    L._check(load().uft_copy(handle, len(s), _at(s), _at(d), stream))


def uft_keep(handle, seqs, starts, counts, index=None, stream=None) -> None:
    s, a, c = ints(seqs), ints(starts), ints(counts)
    _same(s, a, "seqs and starts")
    _same(s, c, "seqs and counts")
    L._check(load().uft_keep(handle, len(s), _at(s), _at(a), _at(c), L._ptr(index), stream))


def uft_trim(handle, seqs, window, sinks, stream=None) -> None:
    s = ints(seqs)
    L._check(load().uft_trim(handle, len(s), _at(s), window, sinks, stream))


def uft_free(handle, seqs) -> None:
    s = ints(seqs)
    L._check(load().uft_free(handle, len(s), _at(s)))


def uft_pack(handle, stream=None) -> int:
    out = _I()
    L._check(load().uft_pack(handle, _ref(out), stream))
    return out.value


def uft_get_info(handle) -> uft_info:
    info = uft_info()
    L._check(load().uft_get_info(handle, _ref(info)))
    return info


def uft_seq_tokens(handle, seq) -> int:
    out = _I()
    L._check(load().uft_seq_tokens(handle, seq, _ref(out)))
    return out.value


def uft_seq_pages(handle, seq):
    n = _I()
    L._check(load().uft_seq_pages(handle, seq, None, 0, _ref(n)))
    pages = (_I * n.value)()
    L._check(load().uft_seq_pages(handle, seq, pages, n.value, _ref(n)))
    return list(pages)


def uft_attn_work_bytes(handle, desc) -> int:
    out = _Z()
    L._check(load().uft_attn_work_bytes(handle, _ref(desc), _ref(out)))
    return out.value


def uft_attn(handle, layer, desc, q, tree, o, lse, work, work_bytes=None, stream=None) -> None:
    n = work_bytes if work_bytes is not None else (0 if work is None else work.numel() * work.element_size())
    L._check(load().uft_attn(handle, layer, _ref(desc), L._ptr(q), L._ptr(tree), L._ptr(o), L._ptr(lse), L._ptr(work), n,
                             stream))


def uft_window_fwd(desc, q, k, v, lengths, o, lse, stream=None) -> None:
    L._check(load().uft_window_fwd(_ref(desc), L._ptr(q), L._ptr(k), L._ptr(v), L._ptr(lengths), L._ptr(o), L._ptr(lse),
                                   stream))


def uft_window_bwd_work_bytes(desc) -> int:
    out = _Z()
    L._check(load().uft_window_bwd_work_bytes(_ref(desc), _ref(out)))
    return out.value


def uft_window_bwd(desc, q, k, v, o, lse, do, lengths, dq, dk, dv, work, work_bytes=None, stream=None) -> None:
    n = work_bytes if work_bytes is not None else (0 if work is None else work.numel() * work.element_size())
    L._check(load().uft_window_bwd(_ref(desc), L._ptr(q), L._ptr(k), L._ptr(v), L._ptr(o), L._ptr(lse), L._ptr(do),
                                   L._ptr(lengths), L._ptr(dq), L._ptr(dk), L._ptr(dv), L._ptr(work), n, stream))
