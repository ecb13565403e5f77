"""Long walks of linear attention against the float64 oracle, by the bounds of oracle/states.py: sequences that are not cut, of
nine chunks and more, so that M passes several periods of four chunks, and parts of several periods.  Each case asserts how it
is cut.  Heads are independent of each other: the oracle takes some of each sequence's, one of every decay."""

import pytest
import torch

from oracle import states as O
from tests.gpu_common import f64, require_gpu
from tests.test_gpu_states import D, SCALE, _sizes_attend, check_backward, check_forward, draw, within

pytestmark = pytest.mark.gpu

CHUNK = 32
# nothing forgotten, long and short memories, the last decay with periods of four chunks (e^(128 g) > 1e-13), the first without
DECAYS = [-0.05, 0.0, -0.2, -0.233, -0.235, -2e-4, -1.0, -5.0, -0.002]


def decays(heads):
    return torch.tensor([DECAYS[h % len(DECAYS)] for h in range(heads)], dtype=torch.float32, device="cuda")


def cut(P, q, k, v, g):
    """Parts of a sequence, forwards and backwards."""
    S, desc = P.states.S, P.states._linear_desc(q, k, v, g, None, None)
    state = k.shape[0] * k.shape[2] * D * D * 4
    return max(S.ufs_linear_work_bytes(desc) // state, 1), max(S.ufs_linear_bwd_work_bytes(desc) // (2 * state), 1)


def heads_of(t, heads, group=1):
    """[n, heads, D] of these key heads, or of their query heads, in float64."""
    return f64(t[:, [h * group + i for h in heads for i in range(group)]])


def check_some(P, q, k, v, do, g, lengths, state, dfinal, picks):
    """Both passes; ``picks``: (sequence, key heads) that the oracle takes."""
    B, n, Hk, _ = k.shape
    G = q.shape[2] // Hk
    lens = None
    if lengths is not None:                              # padding may hold anything
        lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for b, m in enumerate(lengths):
            for t in (q, k, v, do):
                t[b, m:] = float("nan")
    o, final = P.linear_attention(q, k, v, g, lengths=lens, state=state, final=True)
    got = P.linear_attention_bwd(q, k, v, do, g, lengths=lens, state=state, dfinal=dfinal)
    torch.cuda.synchronize()
    assert all(t.isfinite().all() for t in (o, final, *got))
    for b, heads in picks:
        m = n if lengths is None else lengths[b]
        name = f"{(B, n, Hk, G)} sequence {b} of {m}"
        for t in (o, *got[:3]):
            assert not t[b, m:].any(), name
        cq, ck, cv, cdo = (heads_of(t[b, :m], heads, w) for t, w in ((q, G), (k, 1), (v, 1), (do, G)))
        s, df = (None if t is None else f64(t[b, heads]) for t in (state, dfinal))
        check_forward(cq, ck, cv, f64(g[heads]), SCALE, heads_of(o[b, :m], heads, G), s, f64(final[b, heads]), name)
        back = [heads_of(t[b, :m], heads, w) for t, w in zip(got[:3], (G, 1, 1))] + [f64(t[b, heads]) for t in got[3:]]
        check_backward(cq, ck, cv, cdo, f64(g[heads]), SCALE, back, s, df, name)


ALL = list(range(len(DECAYS)))
WALKS = [
    # batch, tokens, key heads, group, lengths, carry, the oracle's (sequence, key heads)
    (3, 1100, 64, 1, None, False, [(0, ALL)]),
    (3, 1100, 64, 1, None, True, [(2, ALL)]),
    # the last chunk in every place of its period, full and not
    (4, 416, 64, 1, [416, 385, 353, 320], True, [(0, ALL), (1, ALL), (2, ALL), (3, ALL)]),
    (4, 416, 64, 1, [288, 300, 0, 415], False, [(0, ALL), (1, ALL), (3, ALL)]),
    # several query heads: two an item forwards, and three, an item of one head
    (3, 600, 64, 2, [600, 321, 33], True, [(0, ALL), (1, [0, 2, 5])]),
    (4, 500, 64, 3, None, True, [(1, [0, 1, 3, 4, 8])]),
    (4, 420, 64, 5, [420, 1, 389, 400], False, [(0, [0, 2, 5]), (2, [0, 3, 4])]),
]


@pytest.mark.parametrize("B,n,Hk,G,lengths,carry,picks", WALKS)
def test_walks_that_are_not_cut(B, n, Hk, G, lengths, carry, picks):
    P = require_gpu()
    q, k, v, do = (draw((B, n, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G)))
    g = decays(Hk)
    assert cut(P, q, k, v, g) == (1, 1) and n > 9 * CHUNK
    state, dfinal = (draw((B, Hk, D, D), i, dtype=torch.float32) if carry else None for i in (8, 9))
    check_some(P, q, k, v, do, g, lengths, state, dfinal, picks)


PARTS = [
    # batch, tokens, key heads, group, parts (of a period or more each), the oracle's: each walk sums the parts before it,
    (1, 2000, 64, 1, (4, 1), [(0, [0, 2, 3, 5])]),
    (2, 2000, 32, 2, (8, 4), [(1, [0, 1, 3])]),
    # and carried on by a launch of their own
    (1, 2000, 16, 3, (16, 9), [(0, [0, 3, 4])]),
]


@pytest.mark.parametrize("B,n,Hk,G,parts,picks", PARTS)
def test_parts_of_several_periods(B, n, Hk, G, parts, picks):
    P = require_gpu()
    q, k, v, do = (draw((B, n, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G)))
    g = decays(Hk)
    assert cut(P, q, k, v, g) == parts
    state, dfinal = (draw((B, Hk, D, D), i, dtype=torch.float32) for i in (8, 9))
    check_some(P, q, k, v, do, g, None, state, dfinal, picks)


@pytest.mark.parametrize("Hk,G,counts", [(64, 1, [(1100, 800, 700), (321, 3, 290)]), (64, 2, [(600, 600, 600), (1, 300, 545)])])
def test_steps_that_are_not_cut(Hk, G, counts):
    """Prompts, and pieces over the states that they leave."""
    P = require_gpu()
    seqs, heads = [2, 0, 1], [0, 1, 2, 3, 4]
    cache, g = P.StateCache(1, Hk, 3), decays(Hk)
    cache.pool.view(torch.int32).fill_(0x7FC00000)
    held = {s: (None, None, 0) for s in seqs}
    for i, step in enumerate(counts):
        cache.extend(seqs, step)
        assert cache.work_bytes() == 0 and max(step) > 9 * CHUNK
        n = sum(step)
        q, k, v = (draw((n, h, D), 3 * i + j) for j, h in enumerate((Hk * G, Hk, Hk)))
        o = cache.attention(0, q, k, v, g)
        torch.cuda.synchronize()
        at = 0
        for s, m in zip(seqs, step):
            args = [heads_of(t[at:at + m], heads, w) for t, w in ((q, G), (k, 1), (v, 1))]
            state, size, total = held[s]
            want, last = O.attend(*args, f64(g[heads]), SCALE, state)
            scope, scope_last = _sizes_attend(*args, f64(g[heads]), SCALE, size)
            name = f"step {i} sequence {s}"
            within("o", heads_of(o[at:at + m], heads, G), want, O.bf16_bound(want, scope, total + m), name)
            within("state", f64(cache.states_view()[0, s, heads]), last, O.fp32_bound(scope_last, total + m), name)
            held[s] = (last, scope_last, total + m)
            at += m


def test_small_gradients_keep_their_bits_through_whole_periods():
    """Powers of two pass through every product: results of 2^-60 times v and dO are 2^-60 times their own."""
    P = require_gpu()
    B, n, Hk = 3, 421, 64
    tiny = 2.0 ** -60
    q, k, v, do = (draw((B, n, Hk, D), i) for i in range(4))
    g = decays(Hk)
    assert cut(P, q, k, v, g) == (1, 1) and n > 13 * CHUNK
    o, final = P.linear_attention(q, k, v * tiny, g, final=True)
    got = P.linear_attention_bwd(q, k, v, do * tiny, g)
    torch.cuda.synchronize()
    big, args = 2.0 ** 60, [heads_of(t[1], ALL) for t in (q, k, v, do)]
    check_forward(*args[:3], f64(g[ALL]), SCALE, heads_of(o[1], ALL) * big, None, f64(final[1, ALL]) * big, "forwards")
    check_backward(*args, f64(g[ALL]), SCALE, [heads_of(t[1], ALL) * big for t in got], what="backwards")


@pytest.mark.parametrize("at", [127, 128, 300])
def test_values_that_are_not_finite_in_a_later_period(at):
    """A value that is not finite leaves the tokens before it (dk and dv: behind it) and the other heads as they were."""
    P = require_gpu()
    B, n, Hk = 3, 420, 64
    base = [draw((B, n, Hk, D), i) for i in range(4)]
    g = decays(Hk)
    assert cut(P, *base[:3], g) == (1, 1)

    def run(q, k, v, do):
        return [P.linear_attention(q, k, v, g), *P.linear_attention_bwd(q, k, v, do, g)]

    clean = run(*base)
    for which in range(4):
        for kind in (float("nan"), float("inf")):
            x = [t.clone() for t in base]
            x[which][1, at, 0, 77] = kind
            got = run(*x)
            one, upto, after = slice(at, at + 1), slice(0, at + 1), slice(at, n)
            spoiled = {0: (one, None, upto, upto), 1: (after, after, None, one), 2: (after, after, one, None),
                       3: (None, one, upto, upto)}[which]
            for name, a, b, hit in zip(("o", "dq", "dk", "dv"), got, clean, spoiled):
                same = torch.ones((B, n, Hk), dtype=torch.bool, device="cuda")
                if hit is not None:
                    same[1, hit, 0] = False
                    assert not a[1, hit, 0, 77].isfinite().any(), (which, name)
                assert torch.equal(a[same], b[same]), (which, name)


def test_more_places_than_a_launch_of_the_backward_takes():
    """One token each: o = scale (q.k) v, dq = scale (do.v) k, dk = scale (do.v) q, dv = scale (q.k) do, at every place."""
    P = require_gpu()
    B, Hk = 43900, 64                                    # 2.8 million sequences and heads, of which a launch has 2,796,200
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.randn((B, 1, Hk, D), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    g = decays(Hk)
    got = [P.linear_attention(q, k, v, g), *P.linear_attention_bwd(q, k, v, do, g)]
    torch.cuda.synchronize()
    for at in range(0, B, 1000):
        a, b, c, d = (t[at:at + 1000].double() for t in (q, k, v, do))
        for x, y, z, result in ((a, b, c, got[0]), (d, c, b, got[1]), (c, d, a, got[2]), (b, a, d, got[3])):
            want = SCALE * (x * y).sum(-1, keepdim=True) * z
            a0 = SCALE * (x * y).abs().sum(-1, keepdim=True) * z.abs() * (3 * 2.0 ** -15 + O.steps(1))
            bound = a0 + (want.abs() + a0) * O.BF16 + 1e-30        # (as the oracle's bound of a bf16 result)
            assert ((result[at:at + 1000].double() - want).abs() <= bound).all(), at
