"""Calls of the state operators that need no GPU: what is refused and leaves the handle as it was, what the wrappers hand on,
and when a step ends."""

import array
import ctypes
import os
import re

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2606_09150_amd as pkg
    pkg.load()
    return pkg


def _dry(P, layers=2, kv_heads=3, max_seqs=6):
    return P.StateCache(layers, kv_heads, max_seqs, flags=P._lib.UF_F_DRYRUN)


def _refused(P, call, status=None):
    with pytest.raises(P.UfError) as e:
        call()
    assert status is None or e.value.status == status
    return str(e.value)


def test_every_entry_point_of_the_header_is_exported_and_bound(P):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "ufs.h")).read()
    names = set(re.findall(r"\b(ufs_[a-z_]+)\(", text))
    lib = ctypes.CDLL(P._lib.LIB_PATH)
    assert names == set(P._states._SIGNATURES)
    for name in names:
        assert hasattr(lib, name)


def test_sizes(P):
    S = P._states
    d = S.ufs_desc(2, 3, 128, 6, 0)
    assert S.ufs_pool_bytes(d) == 2 * 6 * 3 * 128 * 128 * 4 and S.ufs_table_bytes(d) == 4 * (4 + 5 * 6)
    for bad in (S.ufs_desc(0, 3, 128, 6, 0), S.ufs_desc(2, 0, 128, 6, 0), S.ufs_desc(2, 3, 128, 0, 0), S.ufs_desc(2, 3, 128, 65536, 0),
                S.ufs_desc(65536, 3, 128, 6, 0), S.ufs_desc(2, 4097, 128, 6, 0), S.ufs_desc(2, 3, 128, 6, 8), S.ufs_desc(2, 3, 0, 6, 0),
                S.ufs_desc(65535, 4096, 128, 65535, 0)):
        _refused(P, lambda: S.ufs_pool_bytes(bad), P._lib.UF_ERR_ARG)
    _refused(P, lambda: S.ufs_pool_bytes(S.ufs_desc(2, 3, 64, 6, 0)), P._lib.UF_ERR_UNSUPPORTED)
    real = S.ufs_desc(1, 1, 128, 1, 0)
    _refused(P, lambda: S.ufs_create(real, None, None), P._lib.UF_ERR_ARG)


def test_steps_and_tokens(P):
    c = _dry(P)
    assert c.info().step_seqs == 0
    _refused(P, lambda: c.attention(0, 3, None, None, None), P._lib.UF_ERR_EMPTY)
    c.extend([4, 0], np.array([200, 100], np.uint8))
    assert (c.info().step_seqs, c.info().step_tokens, c.info().step_longest) == (2, 300, 200)
    assert c.step_tokens() == 300 and c.tokens(4) == 200 and c.tokens(0) == 100 and c.tokens(1) == 0
    c.attention(1, 6, None, None, None)
    for call in (lambda: c.attention(2, 3, None, None, None), lambda: c.attention(-1, 3, None, None, None),
                 lambda: c.attention(0, 4, None, None, None), lambda: c.attention(0, 0, None, None, None),
                 lambda: c.attention(0, 3, None, None, None, scale=float("nan")),
                 lambda: c.attention(0, 3, None, None, None, scale=float("inf"))):
        _refused(P, call, P._lib.UF_ERR_ARG)
    c.extend(array.array("H", [4]), array.array("H", [7]))
    assert c.step_tokens() == 7 and c.tokens(4) == 207
    for seqs, counts in (([0, 0], [1, 1]), ([6], [1]), ([-1], [1]), ([0], [-1]), ([], []), ([4], [2 ** 31 - 100])):
        _refused(P, lambda: c.extend(seqs, counts), P._lib.UF_ERR_ARG)
    with pytest.raises(ValueError):
        c.extend([0, 1], [1])
    for seqs in (b"\0\0\0\0", bytearray(4), torch.zeros(1, dtype=torch.int32)):
        with pytest.raises((TypeError, ValueError)):
            c.extend(seqs, [1])
    assert c.tokens(4) == 207 and c.step_tokens() == 7                # a refused call leaves all as it was
    _refused(P, lambda: c.tokens(6), P._lib.UF_ERR_ARG)
    with pytest.raises(ValueError):
        c.tokens(2 ** 32)


def test_scratch_is_wanted_where_sequences_are_cut(P):
    c = _dry(P, kv_heads=1)
    for counts, cut in (([8], False), ([9], False), ([32] * 6, False), ([5000], True), ([1, 5000, 0], True)):
        c.extend(range(len(counts)), counts)
        assert (c.work_bytes() > 0) == cut, counts
        c.free(range(len(counts)))


def test_what_ends_a_step(P):
    c = _dry(P)
    c.extend([0, 1, 2], [3, 3, 0])
    c.fork([0], [5])
    assert c.info().step_seqs == 3 and c.tokens(5) == 3
    c.fork([0], [2])                                  # the step names it, with no token
    assert c.info().step_seqs == 0 and c.tokens(2) == 3
    c.extend([0, 1], [1, 1])
    c.reorder([2, 5], (1, 2))
    assert c.info().step_seqs == 2
    c.reorder([0, 1], (1, 2))
    assert c.info().step_seqs == 0
    c.extend([0, 1], [1, 1])
    c.free([2])
    assert c.info().step_seqs == 2 and c.tokens(2) == 0
    c.free([1])
    assert c.info().step_seqs == 0 and c.tokens(1) == 0
    _refused(P, lambda: c.work_bytes(), P._lib.UF_ERR_EMPTY)


def test_fork_and_reorder_refuse(P):
    c = _dry(P)
    c.extend([0, 1, 2], [3, 3, 4])
    bad, empty = P._lib.UF_ERR_ARG, P._lib.UF_ERR_EMPTY
    for src, dst, status in (([0], [1], bad), ([0, 0], [3, 3], bad), ([3], [4], empty), ([0], [6], bad), ([9], [4], bad), ([], [], bad)):
        _refused(P, lambda: c.fork(src, dst), status)
    for seqs, shape, status in (([0, 2], (1, 2), bad), ([0, 3], (1, 2), empty), ([0, 0], (1, 2), bad), ([0, 6], (1, 2), bad),
                                ([0, 1], (2, 1), None)):
        if status is None:
            c.reorder(seqs, shape)
        else:
            _refused(P, lambda: c.reorder(seqs, shape), status)
    with pytest.raises(ValueError):
        c.reorder([0, 1, 2], (1, 2))
    with pytest.raises(ValueError):
        c.reorder([0, 1], (2,))
    many = P.StateCache(1, 1, 65, flags=P._lib.UF_F_DRYRUN)
    many.extend(range(65), [1] * 65)
    many.reorder(range(64), (1, 64))
    _refused(P, lambda: many.reorder(range(65), (1, 65)), bad)
    assert c.tokens(0) == 3


def test_descriptions_that_are_refused(P):
    S, st = P._states, P._states.uft_stride
    fine = st(2 ** 20, 128, 128)

    def linear(**change):
        d = dict(batch=2, tokens=100, q_heads=4, kv_heads=2, head_dim=128, scale=0.1, q=fine, k=fine, v=fine)
        d.update(change)
        return S.ufs_linear_desc(*d.values())

    assert S.ufs_linear_work_bytes(linear()) == 0 and S.ufs_linear_bwd_work_bytes(linear()) == 0
    for need in (S.ufs_linear_work_bytes(linear(tokens=5000)), S.ufs_linear_bwd_work_bytes(linear(tokens=5000)) // 2):
        assert need > 0 and need % (2 * 2 * 65536) == 0       # a state for each part of each sequence and key head
    for change in (dict(batch=0), dict(tokens=0), dict(q_heads=3), dict(kv_heads=0), dict(tokens=2 ** 30 + 1), dict(q_heads=2 ** 17, kv_heads=2),
                   dict(scale=float("nan")), dict(scale=float("inf")), dict(q=st(0, 12, 128)), dict(k=st(0, 2 ** 24 + 8, 128)),
                   dict(v=st(0, 128, 2 ** 30 + 8)), dict(q=st(-8, 128, 128)), dict(batch=2 ** 30, kv_heads=4)):
        for f in (S.ufs_linear_work_bytes, S.ufs_linear_bwd_work_bytes):
            _refused(P, lambda: f(linear(**change)), P._lib.UF_ERR_ARG)
    _refused(P, lambda: S.ufs_linear_work_bytes(linear(head_dim=64)), P._lib.UF_ERR_UNSUPPORTED)
    none = (None,) * 9
    _refused(P, lambda: S.ufs_linear_fwd(linear(), *none), P._lib.UF_ERR_ARG)
    _refused(P, lambda: S.ufs_linear_bwd(linear(), *(None,) * 13), P._lib.UF_ERR_ARG)

    def select(**change):
        d = dict(groups=2, beams=4, vocab=1000, k=8, type=0, end=3, group_stride=4000, beam_stride=1000)
        d.update(change)
        return S.ufs_select_desc(*d.values())

    assert S.ufs_select_work_bytes(select()) > 0
    for change in (dict(groups=0), dict(beams=0), dict(beams=65), dict(groups=2 ** 19), dict(vocab=0), dict(vocab=2 ** 24 + 1), dict(k=0),
                   dict(k=65), dict(group_stride=-1), dict(beam_stride=2 ** 40 + 1)):
        _refused(P, lambda: S.ufs_select_work_bytes(select(**change)), P._lib.UF_ERR_ARG)
    _refused(P, lambda: S.ufs_select_work_bytes(select(type=3)), P._lib.UF_ERR_UNSUPPORTED)
    _refused(P, lambda: S.ufs_select(select(), *(None,) * 7), P._lib.UF_ERR_ARG)
    one = torch.zeros(4)
    for end in (-1, 1000):
        text = _refused(P, lambda: S.ufs_select(select(end=end), one, one, one, one, one, one, None), P._lib.UF_ERR_ARG)
        assert "end" in text


def test_tensors_that_are_refused(P):
    """CPU tensors, other types, shapes and records of derivatives never reach the library."""
    q, g = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16), torch.zeros(2)
    for call in (lambda: P.linear_attention(q, q, q, g), lambda: P.linear_attention_bwd(q, q, q, q, g),
                 lambda: P.linear_attention(q[0], q, q, g), lambda: P.beam_select(torch.zeros((1, 1, 5)), torch.zeros((1, 1)), 2),
                 lambda: P.beam_select(torch.zeros((1, 5)), torch.zeros((1, 1)), 2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.linear_attention(q.float(), q, q, g)
    with pytest.raises(TypeError):
        P.beam_select(torch.zeros((1, 1, 5), dtype=torch.float64), torch.zeros((1, 1)), 2)


def test_a_handle_that_goes_leaves_the_last_errors_text(P):
    cache, other = _dry(P), _dry(P)
    text = _refused(P, lambda: other.extend([77], [1]))
    cache.close()
    assert "77" in text and "77" in P._lib.uf_last_error()
