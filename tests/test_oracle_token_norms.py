"""The norms that the token operators' results are held to (oracle/tokens.py): results with exactly the stated roundings are
within them, results with one rounding more, or a small slip, are not."""

import numpy as np
import pytest

from oracle import tokens as O

SHAPES = [(200, 0, 0), (300, 50, 4), (300, 6, 2), (257, 128, 0), (600, 20, 3)]
SCALE = 128 ** -0.5


def inputs(n, window, sinks, seed=0):
    rng = np.random.default_rng(seed)
    q, k, v, do = (O.keep_bits(g * rng.standard_normal((n, 128)), 8) for g in (1.25, 1, 1, 1))
    return q, k, v, do, O.sees(np.arange(n), np.arange(n), window, sinks)


def forward(q, k, v, see):
    before, o = O.rounded_attend(q, k, v, see, SCALE)
    return O.keep_bits(before, 8), O.attend(q, k, v, see, SCALE)[1], before, o


def off(got, want):
    return np.linalg.norm(got - want)


def test_bits_are_kept_as_bf16_keeps_them():
    import torch
    x = np.concatenate([np.random.default_rng(1).standard_normal(20000) * 10.0 ** np.random.default_rng(2).integers(-9, 9, 20000),
                        [0.0, 1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8]]).astype(np.float32).astype(np.float64)
    assert np.array_equal(O.keep_bits(x, 8), torch.from_numpy(x).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("n,window,sinks", SHAPES)
def test_the_forwards_norm(n, window, sinks):
    q, k, v, _, see = inputs(n, window, sinks)
    got, _, before, o = forward(q, k, v, see)
    limit = O.norm_limit(o, before - o)
    assert off(got, o) <= limit < 3e-3 * np.linalg.norm(o)
    for bits in (6, 7):
        worse = O.keep_bits(O.rounded_attend(q, k, v, see, SCALE, bits)[0], 8)
        assert off(worse, o) > limit, bits
    assert off(got * (1 + 2.0 ** -7), o) > limit


@pytest.mark.parametrize("n,window,sinks", SHAPES)
def test_the_gradients_norms(n, window, sinks):
    q, k, v, do, see = inputs(n, window, sinks)
    o, lse = forward(q, k, v, see)[:2]
    want = O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks))
    limits = [O.norm_limit(g) for g in want]
    for g, limit in zip(want, limits):
        assert off(O.keep_bits(g, 8), g) <= limit < 2.5e-3 * np.linalg.norm(g)
    # the slips, and which of dq, dk, dv show them
    for slip, shown in ((dict(ds_bits=(8, 8)), [0]), (dict(ds_bits=(6, 6)), [0, 1]), (dict(ds_bits=(16, 7)), [1]),
                        (dict(ds_off=0.01), [0, 1]), (dict(delta_off=0.03), [0, 1]), (dict(p_bits=7), [2])):
        worse = [O.keep_bits(g, 8) for g in O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks), **slip)]
        for i in shown:
            assert off(worse[i], want[i]) > limits[i], (slip, i, off(worse[i], want[i]) / limits[i])


def test_delta_off_by_one_part_in_a_hundred():
    """Where few keys are seen delta is a large part of dS."""
    n, window, sinks = 300, 6, 2
    q, k, v, do, see = inputs(n, window, sinks)
    o, lse = forward(q, k, v, see)[:2]
    want = O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks))
    worse = O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks), delta_off=0.01)
    for i in (0, 1):
        assert off(O.keep_bits(worse[i], 8), want[i]) > O.norm_limit(want[i])


def test_the_stated_roundings_are_within_the_bounds_of_every_element():
    for n, window, sinks in SHAPES:
        q, k, v, do, see = inputs(n, window, sinks, 3)
        o, lse = forward(q, k, v, see)[:2]
        for got, (want, bound) in zip(O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks)), O.grads(q, k, v, do, see, SCALE)):
            assert (np.abs(O.keep_bits(got, 8) - want) <= bound).all()


@pytest.mark.parametrize("n,window,sinks", SHAPES + [(600, 16, 0), (600, 60, 4), (600, 70, 0), (40, 0, 0)])
def test_the_stated_roundings_against_exact_gradients(n, window, sinks):
    """At most one and a half times what the result's own rounding does (1.7e-3 of its norm), whatever the window."""
    q, k, v, do, see = inputs(n, window, sinks, 5)
    o, lse = forward(q, k, v, see)[:2]
    for x, (want, _) in zip(O.rounded_grads(q, k, v, do, o, lse, see, SCALE, O.few_keys(n, window, sinks)), O.grads(q, k, v, do, see, SCALE)):
        assert off(O.keep_bits(x, 8), want) < 1.5 * off(O.keep_bits(want, 8), want)
