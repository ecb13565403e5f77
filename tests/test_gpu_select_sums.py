"""The sums of a selection's probabilities over long rows: lse against float64, where a row is one slice and where it is many."""

import numpy as np
import pytest
import torch

from tests.gpu_common import log, require_gpu

pytestmark = pytest.mark.gpu


def rows(kind, V, dtype):
    gen = torch.Generator().manual_seed(V)
    if kind == "flat":                               # equal terms, behind some that are larger, which each lane has one of
        x = torch.full((V,), -0.25)
        x[:4096] = 0.5
    elif kind == "rising":                           # the maximum rises all the way, by little
        x = torch.linspace(-1, 1, V)
    elif kind == "far":                              # half of the sum under terms that are all small
        x = torch.full((V,), -float(np.float32(np.log(V))))
        x[V // 2] = 0.0
    else:
        x = 2.5 * torch.randn(V, generator=gen)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["flat", "rising", "far", "random"])
@pytest.mark.parametrize("G,W,V", [(64, 16, 2 ** 22 + 5), (1, 3, 2 ** 24), (2, 1, 300001)])
def test_sums_of_long_rows(G, W, V, kind, dtype):
    """One row for all hypotheses.  1,024 of them are not cut into slices."""
    P = require_gpu()
    row = rows(kind, V, dtype)
    x = row.double().numpy()
    lse = np.log(np.exp(x).sum())
    # A term e^(y - c), c the row's maximum rounded up to an integer: y - c, the product with log2 e and that constant are
    # rounded (0.22 of a half step), so that its exponent is off by 2.22 half steps of |y - c|; exp2 is off by two, sixteen terms
    # are added in fp32, by sums of four and two (six at most), waves', slices' and the rows' sums rounded and weighed by exp2 once each (nine).
    away = (np.exp(x - lse) * (np.ceil(x.max()) - x)).sum()
    off = (2.22 * away + 17) * 2.0 ** -24
    best = x.max() - lse
    # and lse and the score are rounded (the logit is exact, the hypothesis' own score 0)
    tol = off + (np.spacing(np.float32(abs(lse))) + np.spacing(np.float32(abs(best)))) / 2
    logits, scores = row.cuda().expand(G, W, V), torch.zeros((G, W), device="cuda")
    s, p, t = P.beam_select(logits, scores, 1)
    torch.cuda.synchronize()
    worst = np.abs(s.double().cpu().numpy() - best).max()
    log(f"  {(G, W, V)} {kind} {dtype}: off {worst:.2e} of {tol:.2e}")
    assert worst <= tol and not p.any()
