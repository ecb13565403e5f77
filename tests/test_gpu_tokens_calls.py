"""The token operators on the GPU in the calls where they can go wrong beside their ordinary ones: odd arguments, values that
are not finite, gradients at the ends of the range, single units of long walks."""

import numpy as np
import pytest
import torch

from tests.gpu_common import f64, require_gpu
from tests.test_gpu_tokens import D, check_step, draw, poison, read

pytestmark = pytest.mark.gpu


def test_small_integer_counts_are_not_summed_in_their_own_type():
    """300 tokens, whose uint8 sum is 44: tensors of 44 rows are refused, of 300 taken."""
    P = require_gpu()
    cache = P.TokenCache(1, 1, 20, 2, 400, 64)
    poison(cache)
    counts = np.array([200, 100], np.uint8)
    cache.extend([0, 1], counts)
    k, v, q = draw((300, 1, D), 1), draw((300, 1, D), 2), draw((300, 2, D), 3)
    for call in (lambda: cache.write(0, k[:44], v[:44]), lambda: cache.attention(0, q[:44]),
                 lambda: cache.keep([0, 1], [0, 0], counts, torch.zeros(44, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    cache.write(0, k, v)
    out = cache.attention(0, q, lse=True)
    torch.cuda.synchronize()
    check_step(cache, 0, q, out, 0, 0, what="uint8", seqs=[0, 1], counts=[200, 100])
    index = torch.cat([torch.arange(200), torch.arange(100)]).flip(0).to(torch.int32).cuda()
    cache.keep([0, 1], [0, 0], np.array([200, 100], np.uint8), index)
    torch.cuda.synchronize()
    # the positions of both sequences' parts: the first names 99 .. 0, 199 .. 100, the second 99 .. 0
    got = read(cache, 0)[0]
    assert cache.tokens(0) == 200 and np.array_equal(got, f64(k)[[*range(99, -1, -1), *range(199, 99, -1)]])
    assert np.array_equal(read(cache, 1)[0], f64(k)[200:][::-1])
