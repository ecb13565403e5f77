"""The token operators on the GPU in the calls where they can go wrong beside their ordinary ones: odd arguments, values that
are not finite, gradients at the ends of the range, single units of long walks."""

import numpy as np
import pytest
import torch

from tests.gpu_common import f64, log, require_gpu
from tests.test_gpu_tokens import D, check_step, draw, fill, poison, read

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


@pytest.mark.parametrize("new,heads", [(1, 2), (40, 2)])
@pytest.mark.parametrize("split", [False, True])
def test_a_value_that_is_not_finite_reaches_its_rows_whatever_its_weight(new, heads, split):
    """One key outweighs the others by over 150 bits, so that theirs underflow beside it, in its slice and in others."""
    P = require_gpu()
    cache = P.TokenCache(1, 1, 70, 1, 4200, 64)
    poison(cache)
    k, v, q = draw((4000 + new, 1, D), 1), draw((4000 + new, 1, D), 2), draw((new, heads, D), 3, 0.02)
    q += draw((1, 1, D), 4)
    k[3900] = 12 * draw((1, D), 4)                       # 12 |q|^2 / sqrt(128), over 100 = 104 / ln 2 bits
    gain = (f64(q[:, :, :]) @ f64(k[3900, 0])).min() / D ** 0.5 - 20
    assert gain > 105
    for bad, kind in ((100, "nan"), (3899, "nan"), (100, "inf")):
        v2 = v.clone()
        v2[bad] = float(kind)
        fill(cache, [0], [4000], 0, k[:4000], v2[:4000])
        fill(cache, [0], [new], 0, k[4000:], v2[4000:])
        cache.n_cu = 256 if split else 0
        assert (cache.work_bytes(heads) > 0) == split
        o, lse = cache.attention(0, q, lse=True)
        torch.cuda.synchronize()
        assert lse.isfinite().all()
        assert not o.isfinite().any(), (bad, kind, int(o.isfinite().sum()))
        cache.free([0])


@pytest.mark.parametrize("tokens,kv,group,window,sinks", [(300, 2, 3, 6, 2), (1500, 1, 2, 20, 3), (200, 1, 1, 0, 0)])
def test_gradients_scale_with_do_over_the_range_of_bf16(tokens, kv, group, window, sinks):
    """Gradients are linear in dO, and a power of two leaves every rounding as it is: the same bits, times that power, as
    long as neither side leaves bf16's range (2^-126 to 2^128)."""
    P = require_gpu()
    q, do = draw((1, tokens, kv * group, D), 1), draw((1, tokens, kv * group, D), 2)
    k, v = draw((1, tokens, kv, D), 3), draw((1, tokens, kv, D), 4)
    o, lse = P.window_attention(q, k, v, window, sinks)
    want = P.window_attention_bwd(q, k, v, o, lse, do, window, sinks)
    torch.cuda.synchronize()
    for power in (112, 40, -40):
        got = P.window_attention_bwd(q, k, v, o, lse, (do.float() * 2.0 ** power).to(torch.bfloat16), window, sinks)
        torch.cuda.synchronize()
        for name, a, b in zip(("dq", "dk", "dv"), got, want):
            log(f"  2^{power} {name}: largest {float(b.float().abs().max()):.3g}, finite {bool(a.isfinite().all())}")
            assert torch.equal(a.float(), b.float() * 2.0 ** power), (power, name)
