"""Scores that are equal though their logits are not, in any order of places: exact against the oracle.  In each row a logit of 0
stands over others near -30, so that lse is less than 2^-22: it leaves a logit there as it is (half a step is 2^-20 or more), and scores
are one sum in float32 (the 0's own is the hypothesis': half a step of that is 2^-15 or more)."""

import numpy as np
import pytest
import torch

from oracle import states as O
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

# a hypothesis' score at which some adjacent logits near -30 have the same sum, and some have not
TYPES = {"bf16": (torch.bfloat16, -3.0e6), "fp16": (torch.float16, -3.0e5), "fp32": (torch.float32, -1.0e3)}


def ladder(dtype, n):
    """n adjacent values of the type, from about -30 upwards, as float32."""
    step = {torch.bfloat16: 2.0 ** -3, torch.float16: 2.0 ** -6, torch.float32: 2.0 ** -19}[dtype]
    x = np.float32(-30.0) + np.arange(n, dtype=np.float32) * np.float32(step)
    assert (torch.from_numpy(x).to(dtype).float().numpy() == x).all() and len(set(x.tolist())) == n
    return x


def check(P, logits, scores, k, dtype):
    """logits float32 [G, W, V], values of the type; scores float32 [G, W]."""
    got = [x.cpu().numpy() for x in P.beam_select(torch.from_numpy(logits).to(dtype).cuda(), torch.from_numpy(scores).cuda(), k)]
    for g in range(len(logits)):
        assert (np.log(np.exp(logits[g].astype(np.float64)).sum(-1)) < 2.0 ** -22).all()
        for a, b in zip((x[g] for x in got), O.select(logits[g], scores[g], k)):
            assert np.array_equal(a, b.astype(a.dtype)), (g, k, a, b)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("k", [2, 3, 9, 64])
def test_the_smaller_of_two_logits_of_one_score_comes_first(kind, k):
    """k of a larger logit at high places, more than k of a smaller one with the same score at low places, and none below it with
    that score: the smaller ones are wanted, of which a list by logits holds few."""
    P = require_gpu()
    dtype, score = TYPES[kind]
    steps = ladder(dtype, 300)
    sums = np.float32(score) + steps
    at = next(i for i in range(1, 299) if sums[i - 1] < sums[i] == sums[i + 1])
    low, high = steps[at], steps[at + 1]
    V = 9000
    logits = np.full((1, 1, V), steps[0] - 60, np.float32)
    logits[0, 0, 8000] = 0.0
    logits[0, 0, 5:5 + 2 * k] = low
    logits[0, 0, 700:700 + 90 * k:90] = high
    check(P, logits, np.array([[score]], np.float32), k, dtype)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,V,few", [(1, 3000, 2), (3, 9001, 3), (4, 20011, 12), (2, 70001, 300), (8, 5000, 40)])
def test_many_scores_that_are_equal(kind, W, V, few):
    P = require_gpu()
    dtype, score = TYPES[kind]
    rng = np.random.default_rng(V)
    few = min(few, 40) if kind == "bf16" else few          # (up to -25)
    steps = ladder(dtype, few)
    for k in (1, 2, 7, 16, 33, 64):
        G = 3
        logits = steps[rng.integers(0, few, (G, W, V))]
        # some rows: their larger values rare, or behind the others
        logits[1] = np.where(rng.random((W, V)) < 4 * k / V, logits[1], steps[rng.integers(0, max(few // 2, 1), (W, V))])
        logits[2].sort(-1)
        logits[np.arange(G)[:, None], np.arange(W)[None], rng.integers(0, V, (G, W))] = 0.0
        spacing = np.spacing(np.float32(abs(score)))
        scores = (np.float32(score) + spacing * rng.integers(-2, 3, (G, W))).astype(np.float32)
        check(P, logits, scores, k, dtype)
