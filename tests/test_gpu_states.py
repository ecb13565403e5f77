"""The state operators on the GPU against the float64 oracle, within bounds that follow from their roundings
(oracle/states.py): linear attention of whole sequences with its gradient, and over the states that a cache holds."""

import math

import numpy as np
import pytest
import torch

from oracle import states as O
from tests.gpu_common import f64, log, require_gpu

pytestmark = pytest.mark.gpu

D = 128
SCALE = 1 / math.sqrt(D)


def draw(shape, seed, gain=1.0, dtype=torch.bfloat16):
    g = torch.Generator()
    g.manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(dtype).cuda()


def decays(heads, seed=0):
    """Log decays from none at all to nearly everything; float32 values."""
    some = [-0.05, 0.0, -1.0, -0.002, -5.0, -0.3, -2e-4]
    return torch.tensor([some[(h + seed) % len(some)] for h in range(heads)], dtype=torch.float32, device="cuda")


def within(name, got, want, bound, what=""):
    off = np.abs(got - want)
    assert np.isfinite(got).all(), (what, name)
    worst = float((off / bound).max()) if off.size else 0.0
    log(f"  {what} {name}: worst {worst:.3f} of the bound")
    assert worst <= 1.0, (what, name, worst)


def near(name, got, want, least, what=""):
    """Norms: bf16 results are off by their own rounding and little else."""
    own = np.linalg.norm(O.round_bf16(want) - want)
    off = np.linalg.norm(got - want)
    log(f"  {what} {name}: off {off / max(np.linalg.norm(want), 1e-300):.2e}, its own rounding {own / max(np.linalg.norm(want), 1e-300):.2e}")
    assert off <= 1.05 * own + least, (what, name, off, own)


def check_forward(q, k, v, g, scale, o, state=None, final=None, what=""):
    """One sequence, float64 arrays [n, heads, D]; state, final [Hk, D, D]."""
    n = q.shape[0]
    want, last = O.attend(q, k, v, g, scale, state)
    size, size_last = _sizes_attend(q, k, v, g, scale, state)
    within("o", o, want, O.bf16_bound(want, size, n), what)
    near("o", o, want, 2.0 ** -15 * np.linalg.norm(size), what)
    if final is not None:
        within("final", final, last, O.fp32_bound(size_last, n), what)
        assert np.linalg.norm(final - last) <= 1e-6 * np.linalg.norm(size_last), what


def _abs(a):
    return None if a is None else np.abs(a)


def _sizes_attend(q, k, v, g, scale, state):
    return O.attend(np.abs(q), np.abs(k), np.abs(v), g, abs(scale), _abs(state))


def check_backward(q, k, v, do, g, scale, got, state=None, dfinal=None, what=""):
    n, G = q.shape[0], q.shape[1] // k.shape[1]
    want = O.grads(q, k, v, do, g, scale, state, dfinal)
    size = O.grads(np.abs(q), np.abs(k), np.abs(v), np.abs(do), g, abs(scale), _abs(state), _abs(dfinal))
    for name, x, w, s, m in zip(("dq", "dk", "dv"), got, want, size, (n, n * G, n * G)):
        within(name, x, w, O.bf16_bound(w, s, m), what)
        near(name, x, w, 2.0 ** -15 * np.linalg.norm(s), what)
    if len(got) > 3:
        within("dstate", got[3], want[3], O.fp32_bound(size[3], n * G), what)
        assert np.linalg.norm(got[3] - want[3]) <= 1e-6 * np.linalg.norm(size[3]), what


WHOLE = [
    # batch, tokens, key heads, group, lengths, carry
    (1, 1, 1, 1, None, False),
    (2, 2, 2, 1, [1, 2], True),
    (1, 31, 1, 2, None, True),
    (3, 32, 2, 1, [32, 0, 7], True),
    (1, 33, 3, 1, None, False),
    (2, 64, 1, 3, [64, 33], False),
    (1, 97, 2, 5, None, True),
    (2, 300, 2, 1, [300, 256], False),
    (3, 515, 1, 2, [515, 1, 257], True),
    (1, 1100, 7, 1, None, True),                     # every decay
    (2, 800, 1, 4, [0, 799], True),
    (2, 330, 1, 7, [330, 31], True),
    (1, 161, 2, 6, None, False),
    (1, 70, 1, 8, [65], True),
    # cut into parts both ways
    (1, 2500, 1, 1, None, True),
    (3, 1500, 1, 2, [1500, 37, 1409], True),
]


@pytest.mark.parametrize("B,n,Hk,G,lengths,carry", WHOLE)
def test_whole_sequences(B, n, Hk, G, lengths, carry):
    P = require_gpu()
    q, k, v, do = draw((B, n, Hk * G, D), 1), draw((B, n, Hk, D), 2), draw((B, n, Hk, D), 3), draw((B, n, Hk * G, D), 4)
    g = decays(Hk, n)
    state = draw((B, Hk, D, D), 5, dtype=torch.float32) if carry else None
    dfinal = draw((B, Hk, D, D), 6, dtype=torch.float32) if carry else None
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if lens is not None:                             # padding may hold anything
        for b, m in enumerate(lengths):
            for t in (q, k, v, do):
                t[b, m:] = float("nan")
    if n >= 1500:
        desc = P.states._linear_desc(q, k, v, g, None, None)
        assert P.states.S.ufs_linear_work_bytes(desc) and P.states.S.ufs_linear_bwd_work_bytes(desc)
    o, final = P.linear_attention(q, k, v, g, lengths=lens, state=state, final=True)
    got = P.linear_attention_bwd(q, k, v, do, g, lengths=lens, state=state, dfinal=dfinal)
    alone = P.linear_attention(q, k, v, g, lengths=lens, state=state)
    torch.cuda.synchronize()
    assert torch.equal(alone, o)
    gd = f64(g)
    for b in range(B):
        m = n if lengths is None else lengths[b]
        what = f"{(B, n, Hk, G)} sequence {b} of {m}"
        for t in (o, *got[:3]):
            assert not t[b, m:].any(), what          # (NaN would count)
        cut = [f64(t[b, :m]) for t in (q, k, v, do)]
        s = None if state is None else f64(state[b])
        df = None if dfinal is None else f64(dfinal[b])
        check_forward(*cut[:3], gd, SCALE, f64(o[b, :m]), s, f64(final[b]), what)
        check_backward(*cut, gd, SCALE, [f64(t[b, :m]) for t in got[:3]] + [f64(t[b]) for t in got[3:]], s, df, what)


def test_strides_scales_and_given_buffers():
    """Views of one projection [B, n, q, k, v heads, D], of transposed tensors and of one broadcast head."""
    P = require_gpu()
    B, n, Hk, G = 2, 1270, 2, 2
    both = draw((B, n, Hk * G + 2 * Hk, D), 11)
    q, k, v = both[:, :, :Hk * G], both[:, :, Hk * G:Hk * G + Hk], both[:, :, Hk * G + Hk:]
    turned = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v)]
    g, do = decays(Hk, 3), draw((B, n, Hk * G, D), 12)
    want = P.linear_attention(q.contiguous(), k.contiguous(), v.contiguous(), g, scale=-0.3, final=True)
    back = P.linear_attention_bwd(q.contiguous(), k.contiguous(), v.contiguous(), do, g, scale=-0.3)
    for a in ((q, k, v), turned):
        out, last = torch.empty_like(want[0]), torch.empty_like(want[1])
        desc = P.states._linear_desc(*a, g, None, None)
        need = max(P.states.S.ufs_linear_work_bytes(desc), P.states.S.ufs_linear_bwd_work_bytes(desc))
        work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        got = P.linear_attention(*a, g, scale=-0.3, final=last, out=out, work=work)
        assert got[0] is out and got[1] is last
        assert torch.equal(out, want[0]) and torch.equal(last, want[1])
        for x, y in zip(P.linear_attention_bwd(*a, do, g, scale=-0.3, work=work), back):
            assert torch.equal(x, y)
    shared = k[:, :, :1].expand(B, n, Hk, D)
    one = P.linear_attention(q, shared, v, g)
    assert torch.equal(one, P.linear_attention(q, shared.contiguous(), v, g))
    for b in range(B):
        check_forward(f64(q[b]), f64(k[b]), f64(v[b]), f64(g), -0.3, f64(want[0][b]), None, f64(want[1][b]), "scale -0.3")


def test_final_states_over_the_first_ones():
    P = require_gpu()
    q, k, v = draw((2, 600, 1, D), 1), draw((2, 600, 1, D), 2), draw((2, 600, 1, D), 3)
    g, state = decays(1), draw((2, 1, D, D), 4, dtype=torch.float32)
    o, final = P.linear_attention(q, k, v, g, state=state, final=True)
    mine = state.clone()
    o2, final2 = P.linear_attention(q, k, v, g, state=mine, final=mine)
    assert final2 is mine and torch.equal(mine, final) and torch.equal(o, o2)


@pytest.mark.parametrize("decay", [0.0, -1e-4, -float("inf"), -60.0, 0.01])
def test_decays_at_the_ends_of_their_range(decay):
    P = require_gpu()
    n = 1000
    q, k, v, do = (draw((1, n, 1, D), i) for i in range(4))
    g = torch.tensor([decay], device="cuda")
    o, final = P.linear_attention(q, k, v, g, final=True)
    got = P.linear_attention_bwd(q, k, v, do, g, state=torch.zeros_like(final))
    torch.cuda.synchronize()
    args = [f64(t[0]) for t in (q, k, v)]
    check_forward(*args, f64(g), SCALE, f64(o[0]), None, f64(final[0]), f"decay {decay}")
    check_backward(*args, f64(do[0]), f64(g), SCALE, [f64(t[0]) for t in got], None, None, f"decay {decay}")


@pytest.mark.parametrize("at", [0, 31, 32, 300, 599])
@pytest.mark.parametrize("kind", ["nan", "inf", "-inf"])
def test_values_that_are_not_finite_reach_what_sees_them(at, kind):
    P = require_gpu()
    n = 600
    base = [draw((1, n, 2, D), i) for i in range(4)]
    g = torch.tensor([-0.01, -0.3], device="cuda")
    clean = [P.linear_attention(*base[:3], g), *P.linear_attention_bwd(*base, g)]
    before, after = slice(0, at), slice(at, n)
    upto, behind = slice(0, at + 1), slice(at + 1, n)
    for which in range(4):
        x = [t.clone() for t in base]
        x[which][0, at, 1, 77] = float(kind)
        got = [P.linear_attention(*x[:3], g), *P.linear_attention_bwd(*x, g)]
        torch.cuda.synchronize()
        # where (o, dq, dk, dv) have to stay as they were, and where not one value may be finite
        one = slice(at, at + 1)
        spoiled = {0: (one, None, upto, upto), 1: (after, after, None, one),
                   2: (after, after, one, None), 3: (None, one, upto, upto)}[which]
        for name, a, b, hit in zip(("o", "dq", "dk", "dv"), got, clean, spoiled):
            assert torch.equal(a[:, :, 0], b[:, :, 0]), (which, name)      # the other head
            keep = torch.ones(n, dtype=torch.bool)
            if hit is not None:
                keep[hit] = False
                # its own column where the value is what is weighed (v of o, k of dq, q of dk, do of dv), else all of them
                column = {(2, "o"), (1, "dq"), (0, "dk"), (3, "dv")}
                part = a[0, hit, 1, 77] if (which, name) in column else a[0, hit, 1]
                assert not part.isfinite().any(), (which, name)
                if (which, name) in column:
                    rest = torch.arange(D) != 77
                    assert torch.equal(a[0, :, 1][:, rest.cuda()], b[0, :, 1][:, rest.cuda()]), (which, name)
            assert torch.equal(a[0, keep.cuda(), 1], b[0, keep.cuda(), 1]), (which, name)


@pytest.mark.parametrize("G", [2, 3, 5])
@pytest.mark.parametrize("at", [0, 40, 95])
def test_values_that_are_not_finite_and_shared_heads(G, at):
    """A query's value stays with its head and token, a key head's reaches its own query heads only."""
    P = require_gpu()
    n = 110
    q, k, v, do = (draw((1, n, h, D), i) for i, h in enumerate((2 * G, 2, 2, 2 * G)))
    g = torch.tensor([-0.01, -0.3], device="cuda")
    o, (dq, _, _) = P.linear_attention(q, k, v, g), P.linear_attention_bwd(q, k, v, do, g)
    for kind in (math.nan, math.inf):
        for name, t, head, (hit_o, hit_q) in (("q", q, G + 1, ((at, at + 1, G + 1, G + 2, None), None)),
                                              ("k", k, 1, ((at, n, G, 2 * G, None), (at, n, G, 2 * G, 77))),
                                              ("v", v, 1, ((at, n, G, 2 * G, 77), (at, n, G, 2 * G, None))),
                                              ("do", do, G + 1, (None, (at, at + 1, G + 1, G + 2, None)))):
            was = t[0, at, head, 77].item()
            t[0, at, head, 77] = kind
            got = (P.linear_attention(q, k, v, g), P.linear_attention_bwd(q, k, v, do, g)[0])
            t[0, at, head, 77] = was
            for a, b, hit in zip(got, (o, dq), (hit_o, hit_q)):
                same = torch.ones_like(a, dtype=torch.bool)
                if hit is not None:
                    t0, t1, h0, h1, column = hit
                    same[0, t0:t1, h0:h1, column if column is not None else slice(None)] = False
                    assert not a[~same].isfinite().any(), (name, kind)
                assert torch.equal(a[same], b[same]), (name, kind)


# ---- the cache ----------------------------------------------------------------------

def poison(cache):
    cache.pool.view(torch.int32).fill_(0x7FC00000)
    cache.table.view(torch.int32).fill_(0x7FFFFFF)


class Model:
    """The cache's sequences in float64, a layer each."""

    def __init__(self, layers, Hk, seqs):
        self.state = np.zeros((layers, seqs, Hk, D, D))
        self.size = np.zeros_like(self.state)
        self.n = [0] * seqs

    def step(self, cache, layer, seqs, counts, q, k, v, g, o, what=""):
        at, of = 0, f64(o)
        for s, n in zip(seqs, counts):
            rows = slice(at, at + n)
            at += n
            if n == 0:
                continue
            args = [f64(t[rows]) for t in (q, k, v)]
            want, last = O.attend(*args, f64(g), SCALE, self.state[layer, s])
            size, size_last = _sizes_attend(*args, f64(g), SCALE, self.size[layer, s])
            total = self.n[s] + n
            within("o", of[rows], want, O.bf16_bound(want, size, total), f"{what} seq {s}")
            got = f64(cache.states_view()[layer, s])
            within("state", got, last, O.fp32_bound(size_last, total), f"{what} seq {s}")
            assert np.linalg.norm(got - last) <= 1e-6 * np.linalg.norm(size_last)
            self.state[layer, s], self.size[layer, s] = last, size_last
            if layer == self.state.shape[0] - 1:
                self.n[s] = total


STEPS = [
    # key heads, group, steps of (sequences, counts)
    (1, 1, [([0], [1]), ([0], [1]), ([0], [33])]),
    (2, 3, [([2, 0], [5, 8]), ([0, 1, 2], [1, 0, 8]), ([1, 2], [9, 1])]),
    (1, 11, [([0, 1], [3, 2]), ([1], [1])]),                                   # more query heads than a block takes
    (1, 20, [([0, 2], [4, 3]), ([2], [2])]),
    (3, 1, [([0, 1, 2], [700, 1, 33]), ([2, 1, 0], [1, 1, 1]), ([0, 2], [257, 300])]),   # parts; unequal
    (2, 2, [([3, 1], [0, 290]), ([3], [31]), ([3, 1], [2, 70])]),
]


@pytest.mark.parametrize("Hk,G,steps", STEPS)
def test_steps_of_a_cache(Hk, G, steps):
    P = require_gpu()
    layers = 2
    cache, model = P.StateCache(layers, Hk, 4), Model(layers, Hk, 4)
    poison(cache)
    g = decays(Hk, 2)
    for i, (seqs, counts) in enumerate(steps):
        cache.extend(seqs, counts)
        n = sum(counts)
        for layer in range(layers):
            q, k, v = draw((n, Hk * G, D), 9 * i + layer), draw((n, Hk, D), 9 * i + 3 + layer), draw((n, Hk, D), 9 * i + 5 + layer)
            o = cache.attention(layer, q, k, v, g)
            torch.cuda.synchronize()
            model.step(cache, layer, seqs, counts, q, k, v, g, o, f"step {i} layer {layer}")
    untouched = [s for s in range(4) if cache.tokens(s) == 0]
    assert cache.states_view()[:, untouched].isnan().all()


def test_a_sequence_begins_again_after_free():
    P = require_gpu()
    cache, g = P.StateCache(1, 1, 2), decays(1)
    poison(cache)
    q, k, v = draw((40, 1, D), 1), draw((40, 1, D), 2), draw((40, 1, D), 3)
    outs = []
    for counts in ([40, 0], [40, 0]):
        cache.extend([0, 1], counts)
        outs.append((cache.attention(0, q, k, v, g), cache.states_view()[0, 0].clone()))
        cache.free([0])
        assert cache.tokens(0) == 0 and cache.info().step_seqs == 0
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_many_sequences_in_a_step():
    """More than a launch's words hold, some single tokens among them, and one long."""
    P = require_gpu()
    n, Hk = 300, 1
    cache, g = P.StateCache(1, Hk, n), decays(Hk)
    poison(cache)
    seqs = list(range(n - 1, -1, -1))
    counts = [(i * 7) % 12 for i in range(n)]
    counts[137] = 500
    model = Model(1, Hk, n)
    for i in range(2):
        cache.extend(seqs, counts)
        total = sum(counts)
        q, k, v = draw((total, Hk, D), i), draw((total, Hk, D), i + 5), draw((total, Hk, D), i + 9)
        o = cache.attention(0, q, k, v, g)
        torch.cuda.synchronize()
        model.step(cache, 0, seqs, counts, q, k, v, g, o, f"step {i}")
        counts = [1 + (s % 2) for s in range(n)]


def test_fork_and_reorder_move_states():
    P = require_gpu()
    layers, Hk = 3, 2
    cache = P.StateCache(layers, Hk, 9)
    cache.extend([0, 1], [3, 4])
    cache.states_view().copy_(draw((layers, 9, Hk, D, D), 1, dtype=torch.float32))
    was = cache.states_view().clone()
    cache.fork([0, 1, 0], [5, 2, 7])
    assert [cache.tokens(s) for s in (5, 2, 7, 3)] == [3, 4, 3, 0]
    now = cache.states_view()
    assert torch.equal(now[:, [5, 2, 7]], was[:, [0, 1, 0]]) and torch.equal(now[:, [0, 1, 3, 4, 6, 8]], was[:, [0, 1, 3, 4, 6, 8]])


@pytest.mark.parametrize("groups,beams", [(1, 1), (1, 2), (3, 5), (2, 8), (2, 9), (1, 16), (2, 17), (1, 32), (1, 33), (1, 64), (50, 17)])
def test_reorder(groups, beams):
    P = require_gpu()
    n = groups * beams + 1
    cache = P.StateCache(2, 1, n)
    gen = torch.Generator().manual_seed(beams)
    seqs = (torch.randperm(n, generator=gen)[:n - 1]).tolist()
    for kind in ("any", "turn", "same", "one", "out"):
        parents = {"any": torch.randint(0, beams, (groups, beams), generator=gen),
                   "turn": torch.arange(1, beams + 1).remainder(beams).expand(groups, beams),
                   "same": torch.arange(beams).expand(groups, beams),
                   "one": torch.full((groups, beams), beams - 1),
                   "out": torch.randint(-2, beams + 3, (groups, beams), generator=gen)}[kind].contiguous()
        parents[-1, -1] = {"out": 2 ** 31 - 1}.get(kind, parents[-1, -1])
        cache.extend(seqs, [1] * len(seqs))
        data = draw((2, n, 1, D, D), beams + 100, dtype=torch.float32)
        cache.states_view().copy_(data)
        cache.reorder(seqs, parents.to(torch.int32).cuda())
        assert cache.info().step_seqs == 0
        want = data.clone()
        for i, s in enumerate(seqs):
            p = int(parents[i // beams, i % beams])
            if 0 <= p < beams:
                want[:, s] = data[:, seqs[i // beams * beams + p]]
        torch.cuda.synchronize()
        assert torch.equal(cache.states_view(), want), kind
