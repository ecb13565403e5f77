"""The state operators as a program runs them: captured and replayed, on other streams, at far offsets, and together in the
beam search of a model with a layer over states and one over a window."""

import math

import numpy as np
import pytest
import torch

from oracle import states as O
from tests.gpu_common import f64, log, require_gpu
from tests.test_gpu_states import D, SCALE, Model, check_backward, check_forward, decays, draw, poison

pytestmark = pytest.mark.gpu


def captured(run):
    """run(), once for warming up and once into a graph."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    return graph, out


@pytest.mark.parametrize("B,n,Hk,G", [(2, 75, 2, 2), (1, 3000, 1, 2)])
def test_forward_and_backward_from_graphs(B, n, Hk, G):
    """Two graphs that share a workspace, replayed with other values and lengths and eager calls in between."""
    P = require_gpu()
    q, k, v, do = (draw((B, n, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G)))
    g, state, dfinal = decays(Hk, 2), draw((B, Hk, D, D), 8, dtype=torch.float32), draw((B, Hk, D, D), 9, dtype=torch.float32)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    desc = P.states._linear_desc(q, k, v, g, None, lens)
    need = max(P.states.S.ufs_linear_work_bytes(desc), P.states.S.ufs_linear_bwd_work_bytes(desc))
    assert (need > 0) == (n > 1000)
    work = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    kw = dict(lengths=lens, state=state)

    def forth(work=work):
        return P.linear_attention(q, k, v, g, final=True, work=work, **kw)

    def back(work=work):
        return P.linear_attention_bwd(q, k, v, do, g, dfinal=dfinal, work=work, **kw)

    (one, o), (two, d) = captured(forth), captured(back)
    for turn in range(4):
        for i, t in enumerate((q, k, v, do)):
            t.copy_(draw(t.shape, 20 * turn + i))
        lens.copy_(torch.tensor([n, (n * turn) // 3][:B], dtype=torch.int32))
        want = (*forth(None), *back(None))
        for t in (*o, *d):
            t.fill_(7.0)
        if turn % 2:
            torch.cuda.synchronize()
        one.replay()
        two.replay()
        if turn == 2:
            one.replay()
        torch.cuda.synchronize()
        for a, b in zip((*o, *d), want):
            assert torch.equal(a, b), turn


REPLAYED = [
    # key heads, group, sequences, counts: token by token (rows and columns split over waves, and not), in chunks, in parts
    (2, 2, [3, 0], [1, 1]),
    (64, 2, [4, 1, 2, 0, 3], [1, 2, 1, 1, 0]),
    (1, 11, [0, 2], [8, 3]),
    (1, 18, [0, 2], [4, 3]),
    (2, 1, [1, 3, 2], [40, 40, 1]),
    (1, 2, [2, 0, 1], [1300, 1300, 5]),
]


@pytest.mark.parametrize("Hk,G,seqs,counts", REPLAYED)
def test_a_captured_layer_follows_later_steps(Hk, G, seqs, counts):
    P = require_gpu()
    cache, eager = P.StateCache(1, Hk, 5), P.StateCache(1, Hk, 5)
    model = Model(1, Hk, 5)
    poison(cache)
    poison(eager)
    n, g = sum(counts), decays(Hk, 1)
    q, k, v = (draw((n, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk)))
    o = torch.empty_like(q)
    cache.extend(seqs, counts)
    need = cache.work_bytes()
    assert (need > 0) == (max(counts) > 1000)
    guard = torch.full((need + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    graph, _ = captured(lambda: cache.attention(0, q, k, v, g, out=o, work=guard[:need] if need else None))
    assert (guard[need:] == 0x5A).all()
    cache.free(seqs)                                     # (the run before the capture took the tokens already)
    poison(cache)
    for turn in range(4):
        order = list(seqs)
        same = [i for i in range(len(seqs)) if counts[i] == counts[0]]
        if turn % 2:                                     # the same counts in the same places, other sequences; some begin
            for i, j in zip(same, same[1:] + same[:1]):
                order[i] = seqs[j]
            if turn == 3:
                cache.free([order[0]])
                eager.free([order[0]])
                model.state[0, order[0]], model.size[0, order[0]], model.n[order[0]] = 0, 0, 0
        for c in (cache, eager):
            c.extend(order, counts)
        for i, t in enumerate((q, k, v)):
            t.copy_(draw(t.shape, 10 * turn + i))
        o.fill_(7.0)
        if turn % 2:
            torch.cuda.synchronize()
        graph.replay()
        want = eager.attention(0, q, k, v, g)
        torch.cuda.synchronize()
        assert torch.equal(o, want), turn
        held = [s for s in range(5) if cache.tokens(s)]
        assert torch.equal(cache.states_view()[0, held], eager.states_view()[0, held])
        if Hk < 10:
            model.step(cache, 0, order, counts, q, k, v, g, o, f"turn {turn}")


def test_selection_and_reordering_from_a_graph():
    P = require_gpu()
    G, W, V, k = 3, 4, 5001, 4
    logits, scores = draw((G, W, V), 1, 2.0), torch.zeros((G, W), device="cuda")
    done = torch.zeros((G, W), dtype=torch.bool, device="cuda")
    cache = P.StateCache(2, 1, G * W)
    seqs = list(range(G * W - 1, -1, -1))
    cache.extend(seqs, [1] * (G * W))
    work = torch.empty(P.states.S.ufs_select_work_bytes(P._states.ufs_select_desc(G, W, V, k, 0, 7, W * V, V)), dtype=torch.uint8, device="cuda")

    def run():
        got = P.beam_select(logits, scores, k, done, 7, work=work)
        cache.reorder(seqs, got[1])
        return got

    cache.states_view().zero_()
    graph, got = captured(run)
    for turn in range(4):
        logits.copy_(draw(logits.shape, 50 + turn, 2.0))
        scores.copy_(-torch.rand((G, W), generator=torch.Generator().manual_seed(turn)))
        done.copy_(torch.rand((G, W), generator=torch.Generator().manual_seed(turn + 9)) < 0.3)
        data = draw((2, G * W, 1, D, D), turn, dtype=torch.float32)
        cache.states_view().copy_(data)
        want = P.beam_select(logits, scores, k, done, 7)
        if turn % 2:
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn
        moved = data.clone()
        for i, s in enumerate(seqs):
            moved[:, s] = data[:, seqs[i // W * W + int(want[1][i // W, i % W])]]
        assert torch.equal(cache.states_view(), moved), turn


def test_other_streams():
    """Every entry point on a stream that is not the current one."""
    P = require_gpu()
    Hk, G = 2, 2
    q, k, v, do = (draw((2, 700, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G)))
    g = decays(Hk)
    logits, scores = draw((2, 3, 4001), 7), torch.zeros((2, 3), device="cuda")
    parents = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device="cuda")

    def run(stream):
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        got = [*P.linear_attention(q, k, v, g, final=True, stream=stream), *P.linear_attention_bwd(q, k, v, do, g, stream=stream),
               *P.beam_select(logits, scores, 4, stream=stream)]
        cache = P.StateCache(2, Hk, 4)
        for at in (0, 1):
            cache.extend([0, 1], [350, 350] if at == 0 else [1, 3], stream=stream)
            n = cache.step_tokens()
            for layer in range(2):
                got.append(cache.attention(layer, q[at, :n], k[at, :n], v[at, :n], g, stream=stream))
            if at == 0:
                cache.free([1])
                cache.fork([0], [1], stream=stream)
                cache.fork([0, 1], [2, 3], stream=stream)
        cache.free([1, 0])
        cache.extend([0, 1], [350, 350], stream=stream)
        for layer in range(2):
            got.append(cache.attention(layer, q[1, :700], k[1, :700], v[1, :700], g, stream=stream))
        cache.reorder([0, 1, 2, 3], parents, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        return got + [cache.states_view().clone()]

    for a, b in zip(run(torch.cuda.Stream()), run(None)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,n,Hk", [(3, 900, 11), (2, 2000, 32), (80, 700, 4), (1, 9000, 2)])
def test_states_exchanged_in_place(B, n, Hk):
    """Final states over the first ones, for few parts and for many, and more of them than run at once: no part's walk may read what
    the last one's has put there."""
    P = require_gpu()
    q, k, v = (draw((B, n, h, D), i) for i, h in enumerate((Hk, Hk, Hk)))
    g = torch.full((Hk,), -1e-3, device="cuda")
    state = draw((B, Hk, D, D), 8, 30.0, dtype=torch.float32)
    want = P.linear_attention(q, k, v, g, state=state, final=True)
    cache = P.StateCache(1, Hk, B)
    for _ in range(3):
        own = state.clone()
        o, final = P.linear_attention(q, k, v, g, state=own, final=own)
        assert torch.equal(o, want[0]) and torch.equal(final, want[1])
        cache.free(list(range(B)))
        cache.extend(list(range(B)), [1] * B)            # (its states count from here on)
        cache.states_view()[0].copy_(state)
        cache.extend(list(range(B)), [n] * B)
        o = cache.attention(0, q.view(-1, Hk, D), k.view(-1, Hk, D), v.view(-1, Hk, D), g)
        assert torch.equal(o.view_as(want[0]), want[0]) and torch.equal(cache.states_view()[0], want[1])


def test_steps_without_tokens():
    P = require_gpu()
    cache, g = P.StateCache(1, 2, 3), decays(2)
    poison(cache)
    none = draw((0, 2, D), 1)
    cache.extend([1, 0], [0, 0])
    assert cache.attention(0, none, none, none, g).shape == (0, 2, D) and cache.tokens(1) == 0
    assert cache.states_view().isnan().all()


def test_lengths_out_of_range_are_brought_into_it():
    P = require_gpu()
    q, k, v, do = (draw((3, 70, 1, D), i) for i in range(4))
    g = decays(1)
    outs = []
    for lens in ([70, 0, 70], [2 ** 31 - 1, -5, 71]):
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        outs.append((*P.linear_attention(q, k, v, g, lengths=n, final=True), *P.linear_attention_bwd(q, k, v, do, g, lengths=n)))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_each_result_is_linear_in_its_arguments():
    """O is linear in q, k, v and the first states each, so differences of any width are its derivatives: <O(.., r, ..), dO> =
    <r, gradient>, and the same of the final states.  Either side is a sum of roundings' errors that are independent, none over
    half a bf16 step of its term: eight times the root of their squares covers them (Hoeffding: but for one case in 10^13)."""
    P = require_gpu()
    B, n, Hk, G = 2, 410, 2, 3
    q, k, v, do = (draw((B, n, h, D), i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G)))
    state, dfinal = draw((B, Hk, D, D), 8, dtype=torch.float32), draw((B, Hk, D, D), 9, dtype=torch.float32)
    g, lens = torch.tensor([-0.03, -0.5], device="cuda"), torch.tensor([n, 333], dtype=torch.int32, device="cuda")
    for t in (q, k, v, do):
        t[1, 333:] = 0
    zero, none = torch.zeros_like(state), torch.zeros_like(do)
    grads = P.linear_attention_bwd(q, k, v, do, g, lengths=lens, state=zero)
    of_final = P.linear_attention_bwd(q, k, v, none, g, lengths=lens, state=zero, dfinal=dfinal)

    def sums(a, b):
        x = a.double() * b.double()
        return float(x.sum()), float(x.square().sum())

    for at, name in enumerate(("dq", "dk", "dv", "dstate")):
        r = draw((q, k, v, state)[at].shape, 30 + at, dtype=(q, k, v, state)[at].dtype)
        if at < 3:
            r[1, 333:] = 0
        args = [r if i == at else t for i, t in enumerate((q, k, v if at < 3 else torch.zeros_like(v), zero))]
        o, final = P.linear_attention(*args[:3], g, lengths=lens, state=args[3], final=True)
        for what, (left, sq_l), (right, sq_r) in (("o", sums(o, do), sums(r, grads[at])), ("final", sums(final, dfinal), sums(r, of_final[at]))):
            # (two bf16 parts of what products read, and fp32 sums, are off by less than a sixteenth of a half step's size)
            tol = 8 * 2.0 ** -8 * math.sqrt(sq_l + sq_r)
            if name == "dq" and what == "final":         # (the final states do not depend on q)
                assert not of_final[0].any()
                continue
            log(f"  {name} by {what}: {left:.6e} {right:.6e}, off {abs(left - right):.2e} of {tol:.2e}")
            assert abs(left - right) <= tol and abs(left) > 0, (name, what)


@pytest.mark.parametrize("decay", [-0.2, -0.3, -0.45, -1.0])
def test_small_gradients_keep_their_bits(decay):
    """Powers of two pass through every product: gradients of 2^-60 times dO are 2^-60 times its own."""
    P = require_gpu()
    n = 230
    q, k, v, do = (draw((1, n, h, D), i) for i, h in enumerate((2, 1, 1, 2)))
    g = torch.tensor([decay], device="cuda")
    got = P.linear_attention_bwd(q, k, v, do * 2.0 ** -60, g)
    check_backward(*(f64(t[0]) for t in (q, k, v, do)), f64(g), SCALE, [f64(t[0]) * 2.0 ** 60 for t in got], what=f"decay {decay}")
    o, final = P.linear_attention(q, k, v * 2.0 ** -60, g, final=True)
    check_forward(*(f64(t[0]) for t in (q, k, v)), f64(g), SCALE, f64(o[0]) * 2.0 ** 60, None, f64(final[0]) * 2.0 ** 60, f"decay {decay}")


def test_far_offsets():
    """A pool of more than 2^31 floats, tokens 2^24 elements apart and logits beyond 2^32: the same bits as near ones."""
    P = require_gpu()
    far, near, g = P.StateCache(4, 1, 40000), P.StateCache(4, 1, 8), decays(1)
    seqs = {far: [39999, 17, 39990, 5], near: [7, 0, 6, 1]}
    outs = []
    for cache in (far, near):
        s, got = seqs[cache], []
        for i, counts in enumerate(([40, 3], [1, 2], [1400, 300])):
            cache.extend(s[:2], counts)
            q, k, v = (draw((sum(counts), h, D), 5 * i + j) for j, h in enumerate((2, 1, 1)))
            got += [cache.attention(layer, q, k, v, g) for layer in range(4)]
        cache.fork([s[0], s[0]], s[2:])
        cache.extend([s[2]], [1])
        got += [cache.attention(3, q[:1], k[:1], v[:1], g)]
        cache.extend([s[0], s[3]], [1, 1])
        cache.reorder([s[0], s[2], s[3]], torch.tensor([[1, 2, 0]], dtype=torch.int32, device="cuda"))
        outs.append(got + [cache.states_view()[:, s].clone()])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    del far, seqs
    gap, n = 2 ** 24, 300
    room = torch.empty(n * gap, dtype=torch.bfloat16, device="cuda")
    wide = [room[i * 256:].as_strided((1, n, 1, D), (0, gap, D, 1)) for i in range(3)]
    plain = [draw((1, n, 1, D), i) for i in range(3)]
    for a, b in zip(wide, plain):
        a.copy_(b)
    do = draw((1, n, 1, D), 9)
    assert torch.equal(P.linear_attention(*wide, g), P.linear_attention(*plain, g))
    for a, b in zip(P.linear_attention_bwd(*wide, do, g), P.linear_attention_bwd(*plain, do, g)):
        assert torch.equal(a, b)
    del wide
    logits, scores = draw((2, 2, 3001), 4), torch.zeros((2, 2), device="cuda")
    view = room.as_strided((2, 2, 3001), (2 ** 32, 4001, 1))
    view.copy_(logits)
    for a, b in zip(P.beam_select(view, scores, 5), P.beam_select(logits, scores, 5)):
        assert torch.equal(a, b)


def test_a_beam_search_of_a_model_with_states_and_a_window():
    """Prompts into one sequence of each request, forked for the beams, then single tokens: a layer over states, one over a
    window of a token cache, logits, the selection, and both caches reordered.  Then each hypothesis that is left is computed
    from its own tokens alone: its states, its window, and the scores along its way."""
    P = require_gpu()
    groups, beams, V, Hk, G, window, turns, end = 2, 3, 257, 2, 2, 6, 8, 3
    gen = np.random.default_rng(5)
    table = [draw((V, h, D), 40 + i) for i, h in enumerate((Hk * G, Hk, Hk, Hk * G, Hk, Hk))]     # by token: q, k, v of either layer
    head = draw((2 * Hk * G * D, V), 50, 0.02).float()
    g = decays(Hk, 3)
    prompts = [gen.integers(4, V, n).tolist() for n in (41, 41)]
    states, tokens = P.StateCache(1, Hk, groups * beams), P.TokenCache(1, Hk, 60, 2 * groups * beams, 200, 64)
    poison(states)
    names, other = list(range(groups * beams)), list(range(groups * beams, 2 * groups * beams))   # of the token cache, in turn
    first = [i * beams for i in range(groups)]

    def step(at, where, ids):
        """One token or prompt each: (o of the states, o of the window), [tokens, Hk * G, D]."""
        counts = [len(x) for x in ids]
        flat = torch.tensor(sum(ids, []), device="cuda")
        q0, k0, v0, q1, k1, v1 = (t[flat] for t in table)
        states.extend(at, counts)
        a = states.attention(0, q0, k0, v0, g)
        tokens.extend(where, counts)
        tokens.write(0, k1, v1)
        return a, tokens.attention(0, q1, window)

    def logits_of(a, b):
        return (torch.cat([a, b], 1).float().flatten(1) @ head).to(torch.bfloat16)

    a, b = step(first, first, prompts)
    last = torch.tensor([len(prompts[0]) - 1, len(prompts[0]) + len(prompts[1]) - 1], device="cuda")
    logits = logits_of(a[last], b[last])[:, None].expand(groups, beams, V)                        # (stride 0 over the beams)
    spread = [i * beams + w for i in range(groups) for w in range(1, beams)]
    states.fork([s // beams * beams for s in spread], spread)
    tokens.fork([s // beams * beams for s in spread], [names[s] for s in spread])
    scores = torch.full((groups, beams), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    done = torch.zeros((groups, beams), dtype=torch.bool, device="cuda")
    said = [[list(prompts[i]) for _ in range(beams)] for i in range(groups)]                      # what each hypothesis read
    for turn in range(turns):
        before = scores
        scores, parents, ids = P.beam_select(logits, scores, beams, done, end)
        want = [O.select(f64(logits)[i].astype(np.float32), before[i].cpu().numpy(), beams, done[i].cpu().numpy(), end) for i in range(groups)]
        for i in range(groups):
            assert parents[i].tolist() == want[i][1].tolist() and ids[i].tolist() == want[i][2].tolist(), (turn, i)
        states.reorder(list(range(groups * beams)), parents)
        come = [i * beams + w for i in range(groups) for w in parents[i].tolist()]
        tokens.fork([names[s] for s in come], other)
        tokens.free(names)
        names, other = other, names
        said = [[said[i][w] + [t] for w, t in zip(parents[i].tolist(), ids[i].tolist())] for i in range(groups)]
        done = torch.gather(done, 1, parents.long()) | (ids == end)
        a, b = step(list(range(groups * beams)), names, [[t] for t in ids.flatten().tolist()])
        logits = logits_of(a, b).view(groups, beams, V)
    torch.cuda.synchronize()
    gd = f64(g)
    t64 = [f64(t) for t in table]
    for i in range(groups):
        for w in range(beams):
            x, s = said[i][w], i * beams + w
            q0, k0, v0, q1, k1, v1 = (t[x] for t in t64)
            exact, final = O.attend(q0, k0, v0, gd, SCALE)
            size, size_last = O.attend(np.abs(q0), np.abs(k0), np.abs(v0), gd, SCALE)
            assert (np.abs(f64(a)[s] - exact[-1]) <= O.bf16_bound(exact[-1], size[-1], len(x))).all(), (i, w)
            assert (np.abs(f64(states.states_view()[0, s]) - final) <= O.fp32_bound(size_last, len(x))).all(), (i, w)
            assert states.tokens(s) == tokens.tokens(names[s]) == len(x)
            see = np.arange(max(0, len(x) - window), len(x))
            for h in range(Hk * G):
                e = h // G
                z = SCALE * k1[see, e] @ q1[-1, h]
                p = np.exp(z - z.max())
                want = (p / p.sum()) @ v1[see, e]
                # (weights in bf16, then O: a half step each, and a little for fp32's sums)
                assert np.abs(f64(b)[s, h] - want).max() <= 2.0 ** -7 * 1.1 * np.abs(v1[see, e]).max(), (i, w, h)
    assert len({tuple(x) for y in said for x in y}) == groups * beams
