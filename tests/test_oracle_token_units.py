"""Keys and values that name their unit of 32 tokens, so that a unit left out of a long walk, or taken twice, shows in O and
LSE: the check itself, on the CPU."""

import numpy as np
import pytest

from oracle import tokens as O

UNIT, D = 32, 128
SCALE = D ** -0.5


def marked(n):
    """K and V [n, D], of 4,096 units at most: unit u has its own pair of dimensions, u % 64 and 64 + u // 64."""
    u = np.arange(n) // UNIT
    v = np.zeros((n, D))
    v[np.arange(n), u % 64] = 1
    v[np.arange(n), 64 + u // 64 % 64] = 1
    return 4 * v, v                                      # (a key's score: 0.35 of the sum of two of q's elements)


def queries(n, heads, seed=0):
    return O.keep_bits(np.random.default_rng(seed).standard_normal((n, heads, D)), 8)


def expected(q, k, v, see):
    """O and LSE of one head."""
    o, lse, _ = O.attend(q, k, v, see, SCALE)
    return o, lse


def accepted(o, lse, want, want_lse):
    """Every element of O is a sum of positive terms, whose weights are off by a bf16 half step, and rounded once more; LSE is
    off by fp32 roundings of scores below 3, of sums and of a logarithm of at most 12."""
    return bool((np.abs(o - want) <= want * (2 * O.BF16 + 2.0 ** -12)).all() and (np.abs(lse - want_lse) <= 2e-5).all())


@pytest.mark.parametrize("n,hole,window,sinks", [(70001, (20032, 39936), 0, 0), (66000, None, 0, 0), (70001, None, 20000, 300),
                                                 (4200, None, 0, 0)])
def test_any_unit_left_out_or_taken_twice_is_rejected(n, hole, window, sinks):
    k, v = marked(n)
    q = queries(1, 1)[:, 0]
    see = O.sees([n - 1], np.arange(n), window, sinks)
    if hole:
        see[:, hole[0]:hole[1]] = False
    want, lse = expected(q, k, v, see)
    assert accepted(O.keep_bits(want, 8), lse, want, lse)
    p = np.where(see[0], np.exp((q @ k.T)[0] * SCALE), 0.0)
    total, sums = p.sum(), p @ v
    last = None
    for first in range(0, n, UNIT):
        own = slice(first, first + UNIT)
        w, o = p[own].sum(), p[own] @ v[own]
        if w == 0:
            continue
        for sign in (-1, 1):
            t = total + sign * w
            assert not accepted((sums + sign * o) / t, np.log([t]), want, lse) or w < 2e-5 * total, first
            # with the right LSE: O shows it by itself, where the unit has 4 keys or more
            assert not accepted((sums + sign * o) / total, lse, want, lse) or see[0, own].sum() < 4, first
        if last is not None:                             # this unit's values in place of the one before
            assert not accepted((sums - last + o) / total, lse, want, lse) or see[0, own].sum() < 4, first
        last = o
