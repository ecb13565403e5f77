"""The selection of a beam search on the GPU, against the oracle's scores (oracle/states.py)."""

import numpy as np
import pytest
import torch

from oracle import states as O
from tests.gpu_common import log, require_gpu

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def check(logits, scores, k, got, done=None, end=None, what=""):
    """Places by places: scores are the float64 ones of what was selected within fp32's roundings, in order, and nothing
    better was left out."""
    s, p, t = (x.cpu().numpy() for x in got)
    G, W, V = logits.shape
    lf, sf = logits.float().cpu().numpy(), scores.cpu().numpy()
    df = None if done is None else done.cpu().numpy()
    for g in range(G):
        exact = O.candidates(lf[g], sf[g], None if df is None else df[g], end, wide=np.float64).reshape(-1)
        there = ~np.isnan(exact)
        m = min(k, int(there.sum()))
        assert (s[g, m:] == -np.inf).all() and (p[g, m:] == -1).all() and (t[g, m:] == -1).all(), (what, g)
        flat = p[g, :m].astype(np.int64) * V + t[g, :m]
        assert len(set(flat.tolist())) == m and ((flat >= 0) & (flat < W * V)).all(), (what, g)
        # lse in float32 parts summed in float64 (relative 2^-21 covers exp2 of a rounded argument), rounded; two roundings of the score
        size = np.abs(sf[g][np.isfinite(sf[g])]).max(initial=0.0) + np.abs(lf[g][np.isfinite(lf[g])]).max(initial=0.0) + 20
        tol = 2.0 ** -21 + 4 * 2.0 ** -24 * size
        assert (np.abs(s[g, :m] - exact[flat]) <= tol).all(), (what, g, np.abs(s[g, :m] - exact[flat]).max())
        order = list(zip(-s[g, :m], flat))
        assert order == sorted(order), (what, g)
        left = np.where(there, exact, -np.inf)
        left[flat] = -np.inf
        if m == k:
            assert left.max() <= s[g, m - 1] + tol, (what, g)


def random_case(G, W, V, seed, dtype, spread=2.5):
    gen = torch.Generator().manual_seed(seed)
    logits = (spread * torch.randn((G, W, V), generator=gen)).to(dtype)
    scores = -30 * torch.rand((G, W), generator=gen)
    done = torch.rand((G, W), generator=gen) < 0.2
    return logits.cuda(), scores.cuda(), done.cuda()


SHAPES = [
    # groups, beams, vocabulary, k
    (1, 1, 1, 1), (1, 1, 3, 64), (2, 3, 7, 5), (3, 1, 4096, 1), (1, 4, 4097, 4), (2, 2, 9001, 64), (5, 7, 1237, 13),
    (1, 64, 515, 64), (1, 1, 70001, 63), (1, 2, 300000, 16), (300, 4, 999, 8),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("G,W,V,k", SHAPES)
def test_selection(G, W, V, k, kind):
    P = require_gpu()
    logits, scores, done = random_case(G, W, V, G + V, TYPES[kind])
    what = f"{(G, W, V, k)} {kind}"
    check(logits, scores, k, P.beam_select(logits, scores, k), what=what)
    end = V // 2
    check(logits, scores, k, P.beam_select(logits, scores, k, done=done, end=end), done, end, what)
    scores[:, 1:] = -float("inf")                     # the first step of a search
    check(logits, scores, k, P.beam_select(logits, scores, k, done=done.to(torch.uint8), end=end), done, end, what)


@pytest.mark.parametrize("kind", list(TYPES))
def test_equal_scores_go_to_the_lowest_place(kind):
    """All logits equal; few values; beams that are alike: their scores are the same bits."""
    P = require_gpu()
    G, W, V = 2, 3, 20011
    scores = torch.full((G, W), -2.5, device="cuda")
    for k in (1, 16, 64):
        flat = torch.zeros((G, W, V), dtype=TYPES[kind], device="cuda")
        s, p, t = P.beam_select(flat, scores, k)
        assert not p.any() and torch.equal(t, torch.arange(k, dtype=torch.int32, device="cuda").expand(G, k))
        gen = torch.Generator().manual_seed(k)
        row = torch.randint(0, 4, (V,), generator=gen).to(TYPES[kind])
        few = row.expand(G, W, V).contiguous().cuda()
        s, p, t = P.beam_select(few, scores, k)
        top = (row == 3).nonzero().flatten()[:k].to(torch.int32).cuda()
        assert not p.any() and torch.equal(t, top.expand(G, k))
        rare = torch.zeros(V, dtype=TYPES[kind])
        rare[[5, V - 1, 9000]] = 4.0                   # nine places of the best score in three beams
        s, p, t = P.beam_select(rare.expand(G, W, V).cuda(), scores, 9)
        assert torch.equal(t, torch.tensor([5, 9000, V - 1] * 3, dtype=torch.int32, device="cuda").expand(G, 9))
        assert torch.equal(p, torch.tensor([0, 0, 0, 1, 1, 1, 2, 2, 2], dtype=torch.int32, device="cuda").expand(G, 9))


@pytest.mark.parametrize("k", [1, 2, 16])
def test_logits_that_round_to_one_score(k):
    """Logits that rise by an ulp from token to token under a score whose ulp is far larger: the lowest tokens of the same
    rounded score are wanted, though their logits are the smallest."""
    P = require_gpu()
    V = 9000
    logits = torch.full((1, 2, V), -20.0)
    logits[0, 1, 100:100 + 3 * k] = 5.0 + torch.arange(3 * k) * 2.0 ** -21
    logits[0, 0, 200:200 + 3 * k] = 5.0 + torch.arange(3 * k) * 2.0 ** -21
    scores = torch.tensor([[-40000.0, -40000.0]])    # spacing 2^-8: a move of lse by an ulp changes no score but on its border
    want = None
    for nudge in (-1, 0, 1):                         # ... which this case is not on
        c = O.candidates(logits[0].numpy(), scores[0].numpy())
        c2 = (scores[0].numpy()[:, None] + (logits[0].numpy() - np.float32(5 + np.log(3 * k) + nudge * 2e-6))).astype(np.float32)
        tops = np.sort(np.unique(c2[c2 > scores[0, 0].item() - 10]))
        assert len(tops) == 1 and c.max() == tops[0]
        want = tops[0]
    s, p, t = (x.cpu() for x in P.beam_select(logits.cuda(), scores.cuda(), k))
    assert (s == float(want)).all() and not p.any() and torch.equal(t[0], torch.arange(200, 200 + k, dtype=torch.int32))
    s, p, t = (x.cpu() for x in P.beam_select(logits.cuda(), scores.cuda(), 4 * k))
    assert torch.equal(t[0], torch.tensor([*range(200, 200 + 3 * k), *range(100, 100 + k)], dtype=torch.int32))
    assert torch.equal(p[0], torch.tensor([0] * 3 * k + [1] * k, dtype=torch.int32))


@pytest.mark.parametrize("k", [3, 16, 63])
def test_rows_with_many_equal_logits_in_places(k):
    """Lists of very unequal lengths: a few stretches of equal large logits among others, in 200 rows at once."""
    P = require_gpu()
    G, W, V = 50, 4, 9001
    gen = torch.Generator().manual_seed(k)
    logits = torch.randn((G, W, V), generator=gen)
    for g in range(G):
        for w in range(W):
            at, n = (int(torch.randint(0, m, (), generator=gen)) for m in (V - 1500, 1500))
            logits[g, w, at:at + n] = 4.0 + (g % 3)
    logits, scores = logits.cuda(), (-30 * torch.rand((G, W), generator=gen)).cuda()
    first = P.beam_select(logits, scores, k)
    check(logits, scores, k, first)
    for _ in range(20):
        for a, b in zip(P.beam_select(logits, scores, k), first):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", list(TYPES))
def test_sorted_rows(kind):
    """Rising logits pass every bar: lists are cut down again and again."""
    P = require_gpu()
    G, W, V = 2, 2, 40000
    row = torch.linspace(-8, 8, V)
    logits = torch.stack([row, row.flip(0)]).expand(G, W, V).to(TYPES[kind]).contiguous().cuda()
    scores = torch.tensor([[-1.0, -1.0], [-1.0, -3.0]], device="cuda")
    for k in (1, 17, 64):
        check(logits, scores, k, P.beam_select(logits, scores, k), what=f"{kind} {k}")


def test_rows_that_masks_leave_empty_and_values_that_are_not_finite():
    P = require_gpu()
    V, inf, nan = 5000, float("inf"), float("nan")
    logits, scores, _ = random_case(1, 6, V, 3, torch.float32)
    logits[0, 0] = -inf                              # nothing left
    logits[0, 1, 17] = nan                           # no probability can be told
    logits[0, 2, 4000] = inf
    logits[0, 3, :] = -inf
    logits[0, 3, [4, 4999]] = 1.0                    # two left
    logits[0, 4] = torch.finfo(torch.float32).min    # a mask of the lowest value: all equally likely
    scores[0, 5] = nan
    got = P.beam_select(logits, scores, 64)
    check(logits, scores, 64, got)
    assert set(got[1][0].tolist()) <= {3, 4}
    got = P.beam_select(logits[:, :4].contiguous(), scores[:, :4].contiguous(), 5)
    assert got[1][0].tolist() == [3, 3, -1, -1, -1] and got[2][0].tolist() == [4, 4999, -1, -1, -1]
    assert abs(got[0][0, 0].item() - scores[0, 3].item() + np.log(2)) < 1e-6 and got[0][0, 2:].eq(-inf).all()
    scores[:] = -inf
    got = P.beam_select(logits, scores, 3)
    assert got[0].eq(-inf).all() and got[1].eq(-1).all() and got[2].eq(-1).all()


def test_finished_hypotheses_are_not_read():
    P = require_gpu()
    logits = torch.full((1, 3, 3000), float("nan"), device="cuda")
    logits[0, 1] = 0.0
    done = torch.tensor([[True, False, True]], device="cuda")
    scores = torch.tensor([[-1.0, -0.5, -9.0]], device="cuda")
    s, p, t = P.beam_select(logits, scores, 3, done=done, end=7)
    assert p[0].tolist() == [0, 1, 1] and t[0].tolist() == [7, 0, 1] and s[0, 0].item() == -1.0
    logits[0, 1] = -float("inf")
    s, p, t = P.beam_select(logits, scores, 3, done=done, end=7)
    assert p[0].tolist() == [0, 2, -1] and t[0].tolist() == [7, 7, -1] and s[0, :2].tolist() == [-1.0, -9.0]


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_odd_places(kind):
    """Rows that begin anywhere in 16 bytes, the last position of a longer tensor, one row for all beams."""
    P = require_gpu()
    wide, scores, _ = random_case(2, 3, 2 * 1003 + 9, 5, TYPES[kind])
    for off in range(0, 9):
        view = wide[:, :, off:off + 1003]
        want = P.beam_select(view.contiguous(), scores, 11)
        for a, b in zip(P.beam_select(view, scores, 11), want):
            assert torch.equal(a, b), off
    steps = wide.view(2, 1, 3, -1).expand(2, 4, 3, wide.shape[2]).contiguous()
    for a, b in zip(P.beam_select(steps[:, -1], scores, 5), P.beam_select(wide, scores, 5)):
        assert torch.equal(a, b)
    one = wide[:, :1].expand(2, 3, -1)
    for a, b in zip(P.beam_select(one, scores, 5), P.beam_select(one.contiguous(), scores, 5)):
        assert torch.equal(a, b)
    check(one, scores, 5, P.beam_select(one, scores, 5))
