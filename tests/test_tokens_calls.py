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
