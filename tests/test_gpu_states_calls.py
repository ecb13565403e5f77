"""Calls over the states of a cache at the borders of their kernels: steps of few tokens where the waves of a workgroup share a
state, and graphs that are replayed after steps that they do not fit."""

import pytest
import torch

from tests import test_gpu_states as states
from tests import test_gpu_states_runs as runs
from tests.gpu_common import require_gpu
from tests.test_gpu_states import D, decays, draw

pytestmark = pytest.mark.gpu


# Few states: the waves of a workgroup have rows of the same columns, up to 4 tokens and 64 sums of tokens and query heads
FEW = [
    # key heads, group, sequences, counts
    (2, 1, [1], [4]), (1, 16, [0, 2], [4, 3]),       # the last row of k and v; of queries and sums
    (1, 17, [0, 2], [4, 3]), (1, 16, [2], [4]),      # a sum more: columns
    (3, 21, [1, 0], [3, 3]), (63, 1, [0, 3, 2, 1], [1, 4, 2, 3]), (64, 1, [0, 3, 2, 1], [1, 4, 2, 3]),   # 252 and 256 states
    (2, 1, [1], [5]), (1, 16, [0, 2], [5, 3]),       # in chunks
]


@pytest.mark.parametrize("Hk,G,seqs,counts", FEW)
def test_steps_of_few_tokens(Hk, G, seqs, counts):
    """Sequences that begin, and that go on."""
    if Hk < 10:
        states.test_steps_of_a_cache(Hk, G, [(seqs, counts)] * 2)
    runs.test_a_captured_layer_follows_later_steps(Hk, G, seqs, counts)


@pytest.mark.parametrize("first,second", [([2000, 1005], [1505, 1500]), ([1505, 1500], [2000, 1005])])
def test_a_graph_after_a_step_that_is_cut_otherwise(first, second):
    """Sequences whose parts the captured launches do not hold are left as they are, and so is what lies behind the scratch."""
    P = require_gpu()
    Hk, n = 32, 3005
    cache, g = P.StateCache(1, Hk, 2), decays(Hk)
    q, k, v = (draw((n, Hk, D), i) for i in range(3))
    o = torch.empty_like(q)
    cache.extend([0, 1], first)
    need = cache.work_bytes()
    guard = torch.full((need + 2 ** 22,), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN, if it were read)
    graph, _ = runs.captured(lambda: cache.attention(0, q, k, v, g, out=o, work=guard[:need]))
    cache.free([0, 1])
    cache.extend([0, 1], second)
    other = cache.work_bytes()
    assert need and other and need != other
    guard.fill_(0xFF)
    states = cache.states_view()
    states.fill_(3.0)
    o.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert (guard[need:] == 0xFF).all()
    if need < other:
        assert (o == 7.0).all() and (states == 3.0).all()
    else:
        want = cache.attention(0, q, k, v, g)
        torch.cuda.synchronize()
        assert want.isfinite().all() and o.isfinite().all()
