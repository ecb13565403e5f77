"""The state operators' definitions (oracle/states.py) against facts outside themselves: sums written out, central
differences, closed forms, enumerated selections."""

import itertools

import numpy as np
import pytest

from oracle import states as O


def draws(seed, *shapes):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(s) for s in shapes]


@pytest.mark.parametrize("n,Hq,Hk,given", [(1, 1, 1, False), (7, 2, 1, True), (12, 4, 2, True), (9, 3, 3, False)])
def test_forward_is_the_sum_over_earlier_tokens(n, Hq, Hk, given):
    D = 5
    q, k, v, S = draws(n, (n, Hq, D), (n, Hk, D), (n, Hk, D), (Hk, D, D))
    g = np.array([-0.3, 0.0, -2.0])[:Hk]
    o, final = O.attend(q, k, v, g, 0.7, S if given else None)
    for h, t in itertools.product(range(Hq), range(n)):
        e = h // (Hq // Hk)
        want = sum(np.exp(g[e] * (t - j)) * (q[t, h] @ k[j, e]) * v[j, e] for j in range(t + 1))
        if given:
            want = want + np.exp(g[e] * (t + 1)) * q[t, h] @ S[e]
        assert np.allclose(o[t, h], 0.7 * want)
    for e in range(Hk):
        want = sum(np.exp(g[e] * (n - 1 - j)) * np.outer(k[j, e], v[j, e]) for j in range(n))
        assert np.allclose(final[e], want + (np.exp(g[e] * n) * S[e] if given else 0))


def test_a_sequence_in_pieces_is_the_sequence():
    q, k, v = draws(3, (20, 2, 4), (20, 1, 4), (20, 1, 4))
    g = np.array([-0.1])
    o, final = O.attend(q, k, v, g, 1.0)
    a, S = O.attend(q[:7], k[:7], v[:7], g, 1.0)
    b, S = O.attend(q[7:], k[7:], v[7:], g, 1.0, S)
    assert np.allclose(np.concatenate([a, b]), o) and np.allclose(S, final)


def test_without_decay_and_with_all_of_it():
    q, k, v = draws(4, (6, 1, 4), (6, 1, 4), (6, 1, 4))
    o, final = O.attend(q, k, v, np.array([0.0]), 1.0)
    assert np.allclose(final[0], k[:, 0].T @ v[:, 0]) and np.allclose(o[-1, 0], q[-1, 0] @ final[0])
    o, final = O.attend(q, k, v, np.array([-np.inf]), 1.0)
    assert np.allclose(o[:, 0], (q[:, 0] * k[:, 0]).sum(1, keepdims=True) * v[:, 0])


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (4, 2)])
def test_gradients_are_central_differences(Hq, Hk):
    n, D = 6, 3
    q, k, v, S, do, df = draws(5, (n, Hq, D), (n, Hk, D), (n, Hk, D), (Hk, D, D), (n, Hq, D), (Hk, D, D))
    g = np.array([-0.4, -0.05])[:Hk]

    def loss(q, k, v, S):
        o, final = O.attend(q, k, v, g, 0.6, S)
        return (o * do).sum() + (final * df).sum()

    got = O.grads(q, k, v, do, g, 0.6, S, df)
    for i, grad in enumerate(got):
        args = [q, k, v, S]
        for at in np.ndindex(args[i].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[i][at] += 1e-5
            down[i][at] -= 1e-5
            assert abs((loss(*up) - loss(*down)) / 2e-5 - grad[at]) < 1e-7


def test_selection_by_enumeration():
    rng = np.random.default_rng(6)
    for _ in range(30):
        W, V, k = rng.integers(1, 5), rng.integers(1, 7), int(rng.integers(1, 12))
        logits = rng.integers(-2, 3, (W, V)).astype(np.float32)          # many equal ones
        logits[rng.random((W, V)) < 0.2] = -np.inf
        scores = rng.integers(-3, 0, W).astype(np.float32)
        scores[rng.random(W) < 0.2] = -np.inf
        done = rng.random(W) < 0.3
        s, p, t = O.select(logits, scores, k, done, 0)
        every = []
        for w in range(W):
            lse = np.float32(np.log(np.exp(logits[w].astype(float)).sum())) if np.isfinite(logits[w]).any() else None
            for x in range(V):
                if done[w]:
                    c = scores[w] if x == 0 else None
                else:
                    c = None if lse is None else scores[w] + (logits[w, x] - lse)
                if c is not None and c > -np.inf:
                    every.append((-c, w, x))
        every = sorted(every)[:k]
        assert [(a, b, c) for a, b, c in zip(-s, p, t)][:len(every)] == every
        assert (p[len(every):] == -1).all() and (t[len(every):] == -1).all() and (s[len(every):] == -np.inf).all()


def test_selection_takes_no_nan():
    logits = np.array([[np.nan, 1, 2], [np.inf, 1, 2], [0, 1, 2]], np.float32)
    s, p, t = O.select(logits, np.zeros(3, np.float32), 4)
    assert list(p) == [2, 2, 2, -1] and list(t) == [2, 1, 0, -1]


def test_bounds_tell_a_part_too_few():
    """What the bounds allow is below what one bf16 part in the place of two would do to a typical result's sum."""
    (x,) = draws(7, (1000,))
    assert np.abs(O.round_bf16(x) - x).max() <= O.BF16 * np.abs(x).max()
    assert 3 * 2.0 ** -15 + O.steps(300) < 2.0 ** -9 / 4
