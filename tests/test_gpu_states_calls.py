"""Calls over the states of a cache that other calls do not fit: graphs that are replayed after steps of other counts."""

import pytest
import torch

from tests import test_gpu_states_runs as runs
from tests.gpu_common import require_gpu
from tests.test_gpu_states import D, decays, draw

pytestmark = pytest.mark.gpu


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
