"""ctypes binding of the state operators of libuf.so (include/ufs.h): argument marshalling only."""

import ctypes

from . import _lib as L
from ._tokens import _at, _ref, _same, ints, uft_stride

UFS_BF16, UFS_FP16, UFS_FP32 = 0, 1, 2
UFS_MAX_BEAMS = 64


class ufs_desc(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class ufs_info(ctypes.Structure):
    _fields_ = [("step_seqs", ctypes.c_int32), ("step_tokens", ctypes.c_int32), ("step_longest", ctypes.c_int32)]


class ufs_attn_desc(ctypes.Structure):
    _fields_ = [("q_heads", ctypes.c_int32), ("scale", ctypes.c_float), ("q", uft_stride), ("k", uft_stride),
                ("v", uft_stride)]


class ufs_linear_desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q", uft_stride), ("k", uft_stride), ("v", uft_stride)]


class ufs_select_desc(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("beams", ctypes.c_int32), ("vocab", ctypes.c_int32), ("k", ctypes.c_int32),
                ("type", ctypes.c_int32), ("end", ctypes.c_int32), ("group_stride", ctypes.c_int64),
                ("beam_stride", ctypes.c_int64)]


_P, _I, _Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_IP, _ZP = ctypes.POINTER(_I), ctypes.POINTER(_Z)
_SIGNATURES = {
    "ufs_linear_work_bytes": [ctypes.POINTER(ufs_linear_desc), _ZP],
    "ufs_linear_fwd": [ctypes.POINTER(ufs_linear_desc)] + [_P] * 9 + [_Z, _P],
    "ufs_linear_bwd_work_bytes": [ctypes.POINTER(ufs_linear_desc), _ZP],
    "ufs_linear_bwd": [ctypes.POINTER(ufs_linear_desc)] + [_P] * 13 + [_Z, _P],
    "ufs_pool_bytes": [ctypes.POINTER(ufs_desc), _ZP],
    "ufs_table_bytes": [ctypes.POINTER(ufs_desc), _ZP],
    "ufs_create": [ctypes.POINTER(ufs_desc), _P, _Z, _P, _Z, ctypes.POINTER(_P)],
    "ufs_destroy": [_P],
    "ufs_extend": [_P, _I, _P, _P, _P],
    "ufs_attn_work_bytes": [_P, _ZP],
    "ufs_attn": [_P, _I, ctypes.POINTER(ufs_attn_desc)] + [_P] * 6 + [_Z, _P],
    "ufs_fork": [_P, _I, _P, _P, _P],
    "ufs_reorder": [_P, _I, _I, _P, _P, _P],
    "ufs_free": [_P, _I, _P],
    "ufs_get_info": [_P, ctypes.POINTER(ufs_info)],
    "ufs_seq_tokens": [_P, _I, _IP],
    "ufs_select_work_bytes": [ctypes.POINTER(ufs_select_desc), _ZP],
    "ufs_select": [ctypes.POINTER(ufs_select_desc)] + [_P] * 7 + [_Z, _P],
}

_lib = None


def load():
    """libuf.so with the signatures of the state operators."""
    global _lib
    if _lib is None:
        lib = L.load()
        for name, args in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = lib
    return _lib


def _size(call, *args) -> int:
    out = _Z()
    L._check(call(*args, _ref(out)))
    return out.value


def _bytes(work, work_bytes) -> int:
    return work_bytes if work_bytes is not None else (0 if work is None else work.numel() * work.element_size())


def ufs_linear_work_bytes(desc) -> int:
    return _size(load().ufs_linear_work_bytes, _ref(desc))


def ufs_linear_fwd(desc, q, k, v, decay, lengths, state, o, final, work, work_bytes=None, stream=None) -> None:
    p = L._ptr
    L._check(load().ufs_linear_fwd(_ref(desc), p(q), p(k), p(v), p(decay), p(lengths), p(state), p(o), p(final), p(work),
                                   _bytes(work, work_bytes), stream))


def ufs_linear_bwd_work_bytes(desc) -> int:
    return _size(load().ufs_linear_bwd_work_bytes, _ref(desc))


def ufs_linear_bwd(desc, q, k, v, do, decay, lengths, state, dfinal, dq, dk, dv, dstate, work, work_bytes=None,
                   stream=None) -> None:
    p = L._ptr
    L._check(load().ufs_linear_bwd(_ref(desc), p(q), p(k), p(v), p(do), p(decay), p(lengths), p(state), p(dfinal), p(dq),
                                   p(dk), p(dv), p(dstate), p(work), _bytes(work, work_bytes), stream))


def ufs_pool_bytes(desc) -> int:
    return _size(load().ufs_pool_bytes, _ref(desc))


def ufs_table_bytes(desc) -> int:
    return _size(load().ufs_table_bytes, _ref(desc))


def ufs_create(desc, pool, table, pool_bytes=None, table_bytes=None):
    """pool, table: device tensors (or None under UF_F_DRYRUN). Returns the opaque handle."""
    h = _P()
    L._check(load().ufs_create(_ref(desc), L._ptr(pool), _bytes(pool, pool_bytes), L._ptr(table), _bytes(table, table_bytes),
                               _ref(h)))
    return h


def ufs_destroy(handle) -> None:
    L._check(load().ufs_destroy(handle))


def ufs_extend(handle, seqs, counts, stream=None) -> None:
    s, c = ints(seqs), ints(counts)
    _same(s, c, "seqs and counts")
    L._check(load().ufs_extend(handle, len(s), _at(s), _at(c), stream))


def ufs_attn_work_bytes(handle) -> int:
    return _size(load().ufs_attn_work_bytes, handle)


def ufs_attn(handle, layer, desc, q, k, v, decay, o, work, work_bytes=None, stream=None) -> None:
    p = L._ptr
    L._check(load().ufs_attn(handle, layer, _ref(desc), p(q), p(k), p(v), p(decay), p(o), p(work), _bytes(work, work_bytes),
                             stream))


def ufs_fork(handle, src, dst, stream=None) -> None:
    s, d = ints(src), ints(dst)
    _same(s, d, "src and dst")
    L._check(load().ufs_fork(handle, len(s), _at(s), _at(d), stream))


def ufs_reorder(handle, beams, seqs, parents, stream=None) -> None:
    """seqs: group by group, ``beams`` of each."""
    s = ints(seqs)
    if beams < 1 or len(s) % beams:
        raise ValueError(f"{len(s)} sequences are no groups of {beams}")
    L._check(load().ufs_reorder(handle, len(s) // beams, beams, _at(s), L._ptr(parents), stream))


def ufs_free(handle, seqs) -> None:
    s = ints(seqs)
    L._check(load().ufs_free(handle, len(s), _at(s)))


def ufs_get_info(handle) -> ufs_info:
    info = ufs_info()
    L._check(load().ufs_get_info(handle, _ref(info)))
    return info


def ufs_seq_tokens(handle, seq) -> int:
    out = _I()
    L._check(load().ufs_seq_tokens(handle, seq, _ref(out)))
    return out.value


def ufs_select_work_bytes(desc) -> int:
    return _size(load().ufs_select_work_bytes, _ref(desc))


def ufs_select(desc, logits, scores, done, best, parents, tokens, work, work_bytes=None, stream=None) -> None:
    p = L._ptr
    L._check(load().ufs_select(_ref(desc), p(logits), p(scores), p(done), p(best), p(parents), p(tokens), p(work),
                               _bytes(work, work_bytes), stream))
