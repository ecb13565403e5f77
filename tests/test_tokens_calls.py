"""Calls of the token operators that need no GPU: what the wrappers hand on, and when a step ends."""

import array

import numpy as np
import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2606_09150_amd as pkg
    pkg.load()
    return pkg


def _dry(P, n_pages=40, max_seqs=6, max_tokens=700, page=64, layers=2, kv_heads=3):
    return P.TokenCache(layers, kv_heads, n_pages, max_seqs, max_tokens, page, flags=P._lib.UF_F_DRYRUN)


@pytest.mark.parametrize("kind", [np.uint8, np.int16, np.int32, np.int64])
def test_counts_of_any_integer_type_add_up(P, kind):
    """The step's tokens are what the library counts, also where the counts' own type cannot hold their sum."""
    c = _dry(P, n_pages=1200, max_seqs=2, max_tokens=40000)
    counts = np.array([200, 100] if kind is np.uint8 else [20000, 20000], kind)
    c.extend(np.arange(2), counts)
    assert c.step_tokens() == c.info().step_tokens == sum(counts.tolist())
    c.extend([0], array.array("H", [7]))
    assert c.step_tokens() == 7



def test_host_integers_are_counted_as_they_are_handed_on(P):
    c = _dry(P)
    for seqs, counts in (([0, 1, 2, 3], b"\1\0\0\0"), (b"\0\0\0\0", [1]), (bytearray(4), bytearray(4))):
        with pytest.raises((TypeError, ValueError)):
            c.extend(seqs, counts)
        with pytest.raises((TypeError, ValueError)):
            c.keep(seqs, counts, counts, np.zeros(1))
        with pytest.raises((TypeError, ValueError)):
            c.fork(seqs, counts)
    assert c.info().step_seqs == 0 and c.tokens(0) == 0


def test_a_handle_that_goes_leaves_the_last_errors_text(P):
    """Handles are closed whenever Python collects them: also between a failed call and the reader of its text."""
    L = P._lib
    window = P.KVWindow(1, 1, 300, 128, 2, flags=L.UF_F_DRYRUN)
    cache, other = _dry(P), _dry(P)
    for close in (cache.close, window.close):
        with pytest.raises(P.UfError):
            other.extend([77], [1])
        text = L.uf_last_error()
        assert "77" in text
        close()
        assert L.uf_last_error() == text


def _empty(P, *calls):
    for call in calls:
        with pytest.raises(P.UfError) as e:
            call()
        assert e.value.status == P._lib.UF_ERR_EMPTY


def test_a_trim_that_takes_pages_of_the_steps_tokens_ends_the_step(P):
    """The pages go as the window says; what would write or attend tokens without a place is refused then."""
    c = _dry(P, max_tokens=2000)
    c.extend([0, 1], [800, 3])
    c.trim([1], 1)
    c.trim([0], 800)                                   # nothing to give back
    c.write(1, None, None)
    c.attention(1, 6)
    c.trim([0], 737)                                   # page 0, tokens 0 .. 63: all new
    assert c.pages(0) == [-1] + list(range(1, 13)) and c.info().step_seqs == 0 and c.step_tokens() == 0
    _empty(P, lambda: c.write(1, None, None), lambda: c.attention(1, 6), lambda: c.work_bytes(6))
    c.extend([0], [1])
    c.trim([0], 100)                                   # pages of earlier tokens: the step's own are there
    assert c.info().step_seqs == 1 and c.pages(0)[:10] == [-1] * 10 and c.pages(0)[10] >= 0
    c.attention(0, 6)
    # the last page trimmed holds an earlier token and new ones
    c.extend([1], [61])
    c.trim([1], 2)
    assert c.info().step_seqs == 1                     # position 63 of 0 .. 63 is still seen
    c.trim([1], 1)
    assert c.pages(1) == [-1] and c.info().step_seqs == 0
    # a step of sequences that do not grow, and one whose other sequence is trimmed
    c.extend([0], [0])
    c.trim([0], 1)
    assert c.info().step_seqs == 1
    c.extend([2, 3], [1, 200])
    c.trim([2], 1)
    assert c.info().step_seqs == 2
    c.trim([2, 3], 1)
    assert c.info().step_seqs == 0
    assert c.pages(3) == [-1, -1, -1, c.pages(3)[3]] and c.pages(3)[3] >= 0
