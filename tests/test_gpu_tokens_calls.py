"""The token operators on the GPU in the calls where they can go wrong beside their ordinary ones: odd arguments, values that
are not finite, gradients at the ends of the range, single units of long walks."""

import numpy as np
import pytest
import torch

from oracle import tokens as O
from tests import test_oracle_token_units as units
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


def _bad_rows(x, n):
    return ~np.isfinite(x).all(-1)[:n]


def check_gradients_beside(q, k, v, do, grads, window, sinks, n, scale=D ** -0.5):
    """One sequence of n tokens, some of whose rows hold values that are not finite: a gradient is finite, and within the
    bounds, exactly where no such row takes part in it."""
    G = q.shape[1] // k.shape[1]
    see = O.sees(np.arange(n), np.arange(n), window, sinks)
    seen = {"dq": 0, "dk": 0, "dv": 0}
    for hk in range(k.shape[1]):
        sums = {"dk": [0.0, 0.0, np.zeros(n, bool)], "dv": [0.0, 0.0, np.zeros(n, bool)]}
        bk, bv = _bad_rows(k[:, hk], n), _bad_rows(v[:, hk], n)
        kk, vv = np.where(bk[:, None], 0, k[:n, hk]), np.where(bv[:, None], 0, v[:n, hk])
        for h in range(hk * G, (hk + 1) * G):
            bq, bd = _bad_rows(q[:, h], n), _bad_rows(do[:, h], n)
            bad_p = bq | (see & bk).any(1)               # rows whose weights are not finite
            bad_ds = bad_p | bd | (see & bv).any(1)
            args = np.where(bq[:, None], 0, q[:n, h]), kk, vv, np.where(bd[:, None], 0, do[:n, h])
            for name, bad, i in (("dq", bad_ds, 0), ("dk", bad_ds, 1), ("dv", bad_p | bd, 2)):
                want, bound = O.grads(*args, see & ~bad[:, None], scale)[i]
                if name == "dq":
                    got = grads[0][:n, h]
                    assert not np.isfinite(got[bad]).any() and np.isfinite(got[~bad]).all(), (name, h)
                    assert (np.abs(got - want) <= bound)[~bad].all(), (name, h)
                    seen["dq"] += bad.sum()
                else:
                    s = sums[name]
                    s[0], s[1], s[2] = s[0] + want, s[1] + bound, s[2] | (see & bad[:, None]).any(0)
        for name, got in (("dk", grads[1][:n, hk]), ("dv", grads[2][:n, hk])):
            want, bound, bad = sums[name]
            assert not np.isfinite(got[bad]).any() and np.isfinite(got[~bad]).all(), (name, hk)
            assert (np.abs(got - want) <= bound)[~bad].all(), (name, hk)
            seen[name] += bad.sum()
    log(f"  not finite: {seen}")
    return seen


@pytest.mark.parametrize("kind", ["k nan", "v nan", "v inf", "q nan", "do nan", "do inf"])
@pytest.mark.parametrize("tokens,kv,group,window,sinks,length,bad", [
    (400, 2, 3, 40, 5, 400, [130, 131, 300]),
    (333, 1, 5, 0, 0, 300, [250]),                       # no window, padding
    (1500, 1, 2, 20, 3, 1500, [700, 1499]),              # the sinks' rows are cut into parts
    (200, 1, 70, 9, 0, 200, [64, 65]),                   # a group larger than a unit
    (130, 1, 1, 1, 0, 130, [0, 129])])                   # a window of one token
def test_gradients_beside_values_that_are_not_finite(kind, tokens, kv, group, window, sinks, length, bad):
    P = require_gpu()
    x = {"q": draw((2, tokens, kv * group, D), 1), "k": draw((2, tokens, kv, D), 2), "v": draw((2, tokens, kv, D), 3),
         "do": draw((2, tokens, kv * group, D), 4)}
    what, value = kind.split()
    x[what][1, bad, -1] = float(value)                   # of the second sequence's last head
    for t in x.values():
        t[:, length:] = float("nan")
    lengths = torch.full((2,), length, dtype=torch.int32, device="cuda")
    log(f"{kind} tokens={tokens} kv={kv} group={group} window={window} sinks={sinks}")
    o, lse = P.window_attention(x["q"], x["k"], x["v"], window, sinks, lengths=lengths)
    grads = P.window_attention_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], window, sinks, lengths=lengths)
    torch.cuda.synchronize()
    for b in range(2):
        own = [f64(t)[b] for t in (x["q"], x["k"], x["v"], x["do"])]
        seen = check_gradients_beside(*own, [f64(g)[b] for g in grads], window, sinks, length)
        assert (max(seen.values()) > 0) == (b == 1)
        for g in grads:
            assert not g[b, length:].any()


def test_one_element_of_do_that_is_not_finite_stays_in_its_dimension_of_dv():
    P = require_gpu()
    q, do, k, v = (draw((1, 300, 2, D), i) for i in range(4))
    want = P.window_attention_bwd(q, k, v, *P.window_attention(q, k, v, 30), do, 30)[2]
    do[0, 100, 1, 77] = float("nan")
    dv = P.window_attention_bwd(q, k, v, *P.window_attention(q, k, v, 30), do, 30)[2]
    torch.cuda.synchronize()
    hit = torch.zeros_like(dv, dtype=torch.bool)
    hit[0, 71:101, 1, 77] = True
    assert dv[hit].isnan().all() and dv[~hit].isfinite().all()
    near = torch.zeros_like(hit)
    near[0, :, 1] = True                                 # formed again key by key: another order of the sums
    assert torch.equal(dv[~near], want[~near])
    a, b = dv[near & ~hit].float(), want[near & ~hit].float()
    assert (a - b).norm() < 2 ** -7 * b.norm()


def test_tangents_are_refused():
    """Forward-mode derivatives are no more recorded than gradients are."""
    P = require_gpu()
    fwd = torch.autograd.forward_ad
    q, k, v = draw((1, 9, 4, D), 1), draw((1, 9, 2, D), 2), draw((1, 9, 2, D), 3)
    cache = P.TokenCache(1, 2, 8, 1, 100, 64)
    cache.extend([0], [9])
    cache.write(0, k[0], v[0])
    o, lse = P.window_attention(q, k, v)
    with fwd.dual_level():
        dual = [fwd.make_dual(t, torch.ones_like(t)) for t in (q, k, v, o, lse)]
        dq, dk, dv, do, dl = dual
        for call in (lambda: P.window_attention(dq, k, v), lambda: P.window_attention(q, dk, v), lambda: P.window_attention(q, k, dv),
                     lambda: P.window_attention_bwd(q, k, v, do, lse, q), lambda: P.window_attention_bwd(q, k, v, o, dl, q),
                     lambda: P.window_attention_bwd(q, k, v, o, lse, dq), lambda: cache.write(0, dk[0], v[0]),
                     lambda: cache.write(0, k[0], dv[0]), lambda: cache.attention(0, dq[0])):
            with pytest.raises(ValueError):
                call()
        # no tangent, or one that was taken off
        again = P.window_attention(fwd.unpack_dual(dq).primal, k, v)
        assert torch.equal(again[0], o) and torch.equal(cache.attention(0, q[0]), cache.attention(0, fwd.unpack_dual(dq).primal[0]))
    with pytest.raises(Exception):
        torch.func.jvp(lambda x: P.window_attention(x, k, v)[0], (q,), (q,))


@pytest.mark.parametrize("new,heads", [(1, 2), (4, 8), (40, 1), (33, 2)])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("held,hole,page,window,sinks", [
    (70000, (20032, 39936), 64, 0, 0),                   # past a table of 1,024 units and a wave's 64 pages, and a hole
    (66000, None, 128, 0, 0), (70000, None, 64, 20000, 300), (4200, None, 64, 0, 0), (2300, None, 128, 1000, 70)])
def test_every_unit_of_a_long_walk_counts_once(new, heads, split, held, hole, page, window, sinks):
    P = require_gpu()
    n = held + new
    cache = P.TokenCache(1, 1, -(-n // page) + 2, 1, n, page)
    poison(cache)
    k, v = units.marked(n)
    k, v = (torch.from_numpy(x).to(torch.bfloat16)[:, None].cuda() for x in (k, v))
    fill(cache, [0], [held], 0, k[:held], v[:held])
    if hole:
        cache.trim([0], held - hole[1], hole[0])
        assert [p for p, x in enumerate(cache.pages(0)) if x < 0] == list(range(hole[0] // page, hole[1] // page))
    fill(cache, [0], [new], 0, k[held:], v[held:])
    q = units.queries(new, heads, new)
    cache.n_cu = cache.n_cu if split else 0
    for tree in (False, True):
        bits = None
        if tree:                                         # a chain: each new token sees those before it
            bits = torch.tensor([(1 << (t + 1)) - 1 for t in range(new)], dtype=torch.int64, device="cuda")
        log(f"units: {held}+{new} heads={heads} split={split} page={page} window={window} sinks={sinks} tree={tree}")
        assert (cache.work_bytes(heads, window, sinks) > 0) == split
        o, lse = cache.attention(0, torch.from_numpy(q).to(torch.bfloat16).cuda(), window, sinks, tree=bits, lse=True)
        torch.cuda.synchronize()
        see = O.sees(np.arange(held, n), np.arange(n), window, sinks)
        if hole:
            see[:, hole[0]:hole[1]] = False
        for h in range(heads):
            want, wl = units.expected(q[:, h], f64(k)[:, 0], f64(v)[:, 0], see)
            assert units.accepted(f64(o)[:, h], f64(lse)[:, h], want, wl), h


@pytest.mark.parametrize("tokens,kv,group,window,sinks", [(4500, 1, 1, 0, 0), (3000, 2, 3, 700, 130)])
def test_every_unit_of_a_prompt_counts_once(tokens, kv, group, window, sinks):
    """At once through the cache, and as a whole sequence."""
    P = require_gpu()
    k, v = units.marked(tokens)
    q = units.queries(tokens, kv * group)
    kt, vt = (torch.from_numpy(x).to(torch.bfloat16)[:, None].expand(-1, kv, -1).contiguous().cuda() for x in (k, v))
    qt = torch.from_numpy(q).to(torch.bfloat16).cuda()
    cache = P.TokenCache(1, kv, tokens // 64 + 2, 1, tokens, 64)
    poison(cache)
    fill(cache, [0], [tokens], 0, kt, vt)
    out = cache.attention(0, qt, window, sinks, lse=True)
    whole = P.window_attention(qt[None], kt[None], vt[None], window, sinks)
    torch.cuda.synchronize()
    see = O.sees(np.arange(tokens), np.arange(tokens), window, sinks)
    for h in range(kv * group):
        want, lse = units.expected(q[:, h], k, v, see)
        assert units.accepted(f64(out[0])[:, h], f64(out[1])[:, h], want, lse), h
        assert units.accepted(f64(whole[0])[0, :, h], f64(whole[1])[0, h], want, lse), h
