"""The token cache and the attention that reads it, on the GPU, against the float64 oracle: pages bit for bit, attention
within bounds that follow from its roundings (oracle/tokens.py)."""

import math

import numpy as np
import pytest
import torch

from oracle import tokens as O
from tests.gpu_common import f64, log, require_gpu

pytestmark = pytest.mark.gpu

D = 128
SCALE = 1 / math.sqrt(D)


def draw(shape, seed, gain=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(torch.bfloat16).cuda()


def fill(cache, seqs, counts, seed, k=None, v=None, layers=None):
    """Extend and write; returns the new keys and values per layer."""
    cache.extend(seqs, counts)
    out = []
    for layer in range(cache.desc.layers):
        shape = (sum(counts), cache.desc.kv_heads, D)
        kv = (draw(shape, seed + 2 * layer) if k is None else k, draw(shape, seed + 2 * layer + 1) if v is None else v)
        cache.write(layer, *kv)
        out.append(kv)
    return out


def read(cache, seq, layer=0):
    """float64 K, V [tokens, kv_heads, D] of a sequence, through its pages (zeros where trimmed)."""
    n, T = cache.tokens(seq), cache.desc.page_tokens
    pages = cache.pages(seq)
    got = torch.zeros((2, cache.desc.kv_heads, len(pages) * T, D), dtype=torch.bfloat16, device="cuda")
    for i, p in enumerate(pages):
        if p >= 0:
            got[:, :, i * T:(i + 1) * T] = cache.pages_view()[layer, p]
    return f64(got[0, :, :n].permute(1, 0, 2)), f64(got[1, :, :n].permute(1, 0, 2))


def check_rows(q, o, lse, k, v, see, scale=SCALE, what=""):
    """All heads of one sequence: q, o [n, Hq, D], lse [n, Hq] or None, k, v [m, Hk, D] (float64), see [n, m]."""
    G = q.shape[1] // k.shape[1]
    worst = 0.0
    for h in range(q.shape[1]):
        want, wl, p = O.attend(q[:, h], k[:, h // G], v[:, h // G], see, scale)
        # keys that no query sees are left out of the bound
        used = see.any(0)
        kk, vv = k[used, h // G], v[used, h // G]
        if not used.any():
            assert not o[:, h].any()
            continue
        bound = O.attend_bound(q[:, h], kk, vv, p[:, used], want, scale)
        off = np.abs(o[:, h] - want)
        assert np.isfinite(o[:, h]).all(), what
        assert (off <= bound).all(), (what, h, float((off / bound).max()))
        worst = max(worst, float((off / bound).max()))
        empty = ~see.any(1)
        assert not o[empty, h].any()
        if lse is not None:
            assert (lse[empty, h] == -np.inf).all()
            lb = O.lse_bound(q[:, h], kk, wl, scale)
            assert (np.abs(lse[~empty, h] - wl[~empty]) <= lb[~empty]).all(), what
    return worst


def check_step(cache, layer, q, out, window, sinks, bits=None, scale=SCALE, what="", seqs=None, counts=None):
    o, lse = out
    o, lse, qf, at = f64(o), f64(lse), f64(q), 0
    for i, (s, n) in enumerate(zip(seqs, counts)):
        k, v = read(cache, s, layer)
        held = k.shape[0] - n
        see = (O.tree_sees(held, bits[i], window, sinks) if bits is not None
               else O.sees(np.arange(held, held + n), np.arange(held + n), window, sinks))
        T = cache.desc.page_tokens
        for p, page in enumerate(cache.pages(s)):
            if page < 0:
                see[:, p * T:(p + 1) * T] = False
        w = check_rows(qf[at:at + n], o[at:at + n], lse[at:at + n], k, v, see, scale, f"{what} seq {s}")
        log(f"  {what} seq {s}: {n} over {held}, worst {w:.3f} of the bound")
        at += n


def poison(cache):
    """What no sequence holds is never read: NaN everywhere."""
    cache.pool.view(torch.int16).fill_(0x7FC0)
    cache.table.view(torch.int32).fill_(0x7FFFFFF)


CASES = [
    # page, kv heads, group, held, new, window, sinks
    (64, 1, 1, [0], [1], 0, 0),                          # the first token
    (64, 2, 4, [200, 0, 63, 64, 65], [1, 1, 1, 1, 1], 0, 0),
    (128, 3, 5, [1000, 127, 128, 31], [1, 1, 1, 1], 100, 3),
    (64, 1, 32, [777], [1], 65, 70),                     # 32 rows; sinks reach into the window
    (64, 2, 1, [500, 900], [32, 31], 64, 1),             # 32 rows of one head
    (128, 1, 3, [40, 300], [7, 11], 1, 0),               # a window of one token
    (64, 2, 3, [0, 130], [11, 1], 33, 200),              # few rows and many in one step
    (64, 1, 40, [333], [1], 0, 0),                       # more heads than a small tile has rows
    (64, 2, 2, [0], [300], 0, 0),                        # a prompt
    (128, 1, 7, [0, 100, 5], [129, 64, 0], 50, 4),       # heads that do not divide a tile, a sequence that does not grow
    (64, 3, 1, [700, 0], [130, 257], 128, 128),
    (64, 1, 200, [10], [3], 5, 1),                       # a group larger than a tile
    (64, 1, 1, [3000], [150], 1000, 10),                 # cut into slices
]


@pytest.mark.parametrize("page,kv,group,held,new,window,sinks", CASES)
def test_attention_over_the_cache(page, kv, group, held, new, window, sinks):
    P = require_gpu()
    n = len(held)
    cache = P.TokenCache(2, kv, sum(-(-(a + b) // page) for a, b in zip(held, new)) + 3, n + 1, max(held) + max(new), page)
    poison(cache)
    seqs = [(i * 2 + 1) % (n + 1) for i in range(n)] if n % 2 == 0 else list(range(n))
    fill(cache, seqs, held, 1)
    fill(cache, seqs, new, 50)
    for layer in (1, 0):
        q = draw((sum(new), kv * group, D), 99 + layer, 1.5)
        log(f"attend page={page} kv={kv} group={group} {held}+{new} window={window} sinks={sinks}")
        out = cache.attention(layer, q, window, sinks, lse=True)
        torch.cuda.synchronize()
        check_step(cache, layer, q, out, window, sinks, what=f"layer {layer}", seqs=seqs, counts=new)


@pytest.mark.parametrize("kv,group,held,window,sinks,widths", [
    (1, 1, [0, 5], 0, 0, [1, 7]), (2, 4, [100, 64, 200], 0, 0, [8, 3, 8]), (2, 2, [300, 0], 70, 4, [64, 64]),
    (1, 8, [1000], 64, 200, [64]), (3, 1, [2500], 0, 0, [31])])
@pytest.mark.parametrize("page", [64, 128])
def test_tree_over_the_cache(page, kv, group, held, window, sinks, widths):
    P = require_gpu()
    rng = np.random.default_rng(sum(held))
    cache = P.TokenCache(1, kv, 60, 4, 2600, page)
    poison(cache)
    seqs = list(range(len(held)))
    fill(cache, seqs, held, 3)
    fill(cache, seqs, widths, 9)
    bits = []
    for n in widths:
        own = []
        for t in range(n):
            parent = int(rng.integers(-1, t))
            own.append((own[parent] if parent >= 0 else 0) | 1 << t)
        if n > 4:
            own[3] = 0                                   # sees no node
            own[2] |= 1 << (n - 1)                       # sees a later one
            own[1] |= ((1 << 64) - (1 << n)) if n < 64 else 0    # bits of no node
        bits.append(own)
    words = [b - (1 << 64) if b >> 63 else b for own in bits for b in own]
    tree = torch.tensor(words, dtype=torch.int64, device="cuda")
    bits = [[b & ((1 << n) - 1) for b in own] for own, n in zip(bits, widths)]
    q = draw((sum(widths), kv * group, D), 5, 1.5)
    log(f"tree page={page} kv={kv} group={group} {held}+{widths} window={window} sinks={sinks}")
    out = cache.attention(0, q, window, sinks, tree=tree, lse=True)
    torch.cuda.synchronize()
    check_step(cache, 0, q, out, window, sinks, bits, what="tree", seqs=seqs, counts=widths)


def test_split_launches_equal_whole_ones_up_to_rounding():
    P = require_gpu()
    cache = P.TokenCache(1, 2, 80, 2, 4000, 64)
    fill(cache, [0, 1], [3900, 700], 1)
    for new, heads in (([1, 1], 8), ([40, 3], 8)):
        cache.extend([0, 1], new)
        cache.write(0, draw((sum(new), 2, D), 4), draw((sum(new), 2, D), 5))
        q = draw((sum(new), heads, D), 6, 2.0)
        assert cache.work_bytes(heads) > 0
        cut = cache.attention(0, q, lse=True)
        cache.n_cu, n_cu = 0, cache.n_cu
        assert cache.work_bytes(heads) == 0
        whole = cache.attention(0, q, lse=True)
        cache.n_cu = n_cu
        torch.cuda.synchronize()
        check_step(cache, 0, q, cut, 0, 0, what="cut", seqs=[0, 1], counts=new)
        check_step(cache, 0, q, whole, 0, 0, what="whole", seqs=[0, 1], counts=new)


@pytest.mark.parametrize("new,heads", [(1, 2), (40, 1)])
@pytest.mark.parametrize("split", [False, True])
def test_more_keys_than_a_table_of_units_holds(new, heads, split):
    """70,000 tokens, a hole in their middle, whole rows and slices."""
    P = require_gpu()
    cache = P.TokenCache(1, 1, 1200, 1, 70100, 64)
    poison(cache)
    fill(cache, [0], [70000], 1)
    cache.trim([0], 30000, 20000)                        # tokens from 20,032 up to the last 30,000 leave
    fill(cache, [0], [new], 7)
    q = draw((new, heads, D), 3, 2.0)
    cache.n_cu = cache.n_cu if split else 0
    out = cache.attention(0, q, lse=True)
    torch.cuda.synchronize()
    assert cache.pages(0).count(-1) > 300
    check_step(cache, 0, q, out, 0, 0, what="long", seqs=[0], counts=[new])


def test_pages_beyond_four_gigabytes():
    P = require_gpu()
    cache = P.TokenCache(2, 8, 9000, 2, 8900 * 128, 128)  # 4.7 GB a layer
    cache.extend([0], [8890 * 128])                      # takes the low pages, and is never written
    cache.extend([1], [0])
    fill(cache, [1], [400], 3)
    assert min(cache.pages(1)) >= 8890
    for new in (1, 90):
        fill(cache, [1], [new], 20 + new)
        for layer in (0, 1):
            q = draw((new, 16, D), new + layer)
            out = cache.attention(layer, q, 300, 2, lse=True)
            torch.cuda.synchronize()
            check_step(cache, layer, q, out, 300, 2, what=f"layer {layer}", seqs=[1], counts=[new])
    cache.free([0])
    before = [read(cache, 1, layer) for layer in (0, 1)]
    assert cache.pack() == 4 and cache.pages(1) == [0, 1, 2, 3]
    for layer in (0, 1):
        for a, b in zip(before[layer], read(cache, 1, layer)):
            assert np.array_equal(a, b)


def test_large_logits_and_values_behind_the_window():
    """Scores of hundreds, the largest at either end; NaN and infinities where nothing is seen."""
    P = require_gpu()
    cache = P.TokenCache(1, 1, 40, 1, 1100, 64)
    poison(cache)
    k, v = draw((1000, 1, D), 1), draw((1000, 1, D), 2)
    k[[0, 400, 999]] *= 30
    k[10:500] = float("nan")                             # behind a window of 450 and 10 sinks, for tokens from 999 on
    v[10:500] = float("inf")
    fill(cache, [0], [1000], 0, k, v)
    for n, heads in ((1, 4), (1, 40)):
        cache.keep([0], [999], [0])
        cache.extend([0], [n])
        cache.write(0, k[999:], v[999:])
        q = draw((n, heads, D), 3, 3.0)
        q[:, 0] = k[999:, 0] * 0.3
        out = cache.attention(0, q, 450, 10, lse=True)
        kk, vv = read(cache, 0)
        kk[10:500], vv[10:500] = 0, 0
        see = O.sees([999], np.arange(1000), 450, 10)
        assert see[0, :10].all() and not see[0, 10:550].any()
        check_rows(f64(q), f64(out[0]), f64(out[1]), kk, vv, see)


def _only_those_that_see(q, o, lse, k, v, see, bad):
    """Rows that see none of the keys ``bad`` are as if those were anything else; the others are not finite."""
    hit = see[:, bad].any(1)
    assert hit.any() and not hit.all()
    assert not np.isfinite(o[hit]).all(axis=(1, 2)).any()
    if np.isnan(k[bad]).any():
        assert np.isnan(lse[hit]).all()
    k, v = k.copy(), v.copy()
    k[bad], v[bad] = 0, 0
    check_rows(q[~hit], o[~hit], lse[~hit], k, v, see[~hit])


@pytest.mark.parametrize("held,new,heads,window,sinks,bad", [
    (0, 300, 2, 50, 3, [100, 101, 220]),                  # a prompt
    (2000, 40, 1, 0, 0, [2017]),                          # slices
    (500, 3, 8, 60, 2, [502]),                            # few rows
    (90, 8, 4, 0, 0, [97])])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(held, new, heads, window, sinks, bad):
    P = require_gpu()
    for kind in ("v inf", "v nan", "k nan"):
        k, v = draw((held + new, 1, D), 1), draw((held + new, 1, D), 2)
        (k if kind[0] == "k" else v)[bad] = float(kind[2:])
        cache = P.TokenCache(1, 1, 50, 1, 3000, 64)
        poison(cache)
        if held:
            fill(cache, [0], [held], 0, k[:held], v[:held])
        fill(cache, [0], [new], 0, k[held:], v[held:])
        q = draw((new, heads, D), 3)
        log(f"not finite: {kind} {held}+{new} heads={heads}")
        o, lse = cache.attention(0, q, window, sinks, lse=True)
        torch.cuda.synchronize()
        see = O.sees(np.arange(held, held + new), np.arange(held + new), window, sinks)
        _only_those_that_see(f64(q), f64(o), f64(lse), f64(k), f64(v), see, bad)
        bits = [1 << t | (1 if t else 0) for t in range(min(new, 40))]     # a root, and leaves that do not see each other
        if new <= 40:
            words = torch.tensor(bits, dtype=torch.int64, device="cuda")
            o, lse = cache.attention(0, q, window, sinks, tree=words, lse=True)
            torch.cuda.synchronize()
            _only_those_that_see(f64(q), f64(o), f64(lse), f64(k), f64(v), O.tree_sees(held, bits, window, sinks), bad)


def test_strided_views_another_stream_and_the_callers_buffers():
    P = require_gpu()
    cache = P.TokenCache(1, 2, 20, 2, 600, 64)
    qkv = draw((500, 4 + 2 + 2, D), 8)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.extend([0, 1], [450, 50], stream=side)
    cache.write(0, k, v, stream=side)
    o, lse = cache.attention(0, q, 77, 5, lse=True, stream=side)
    side.synchronize()
    check_step(cache, 0, q, (o, lse), 77, 5, what="side stream", seqs=[0, 1], counts=[450, 50])
    torch.cuda.current_stream().wait_stream(side)
    mine = torch.full((500, 4, D), 7.0, dtype=torch.bfloat16, device="cuda")
    back = cache.attention(0, q.contiguous(), 77, 5, out=mine, lse=torch.empty((500, 4), device="cuda"))
    assert back[0] is mine and torch.equal(mine, o) and torch.equal(back[1], lse)
    swapped = torch.empty((2, 500, D), dtype=torch.bfloat16, device="cuda").permute(1, 0, 2)   # heads outermost
    swapped.copy_(k)
    cache.write(0, swapped, v)
    assert torch.equal(cache.attention(0, q, 77, 5), o)


def test_wrappers_refuse():
    P = require_gpu()
    cache = P.TokenCache(1, 2, 8, 2, 100, 64)
    cache.extend([0], [5])
    k, q = draw((5, 2, D), 0), draw((5, 4, D), 0)
    for bad in (k[:4], k.float(), k.cpu(), torch.empty((5, 2, D + 1), dtype=torch.bfloat16, device="cuda")[..., 1:],
                draw((5, 3, D), 0), draw((5, 2, 2 * D), 0)[..., ::2], k.clone().requires_grad_()):
        with pytest.raises((ValueError, TypeError)):
            cache.write(0, k, bad)
        with pytest.raises((ValueError, TypeError)):
            cache.attention(0, bad if bad.shape[0] != 5 or bad.shape[1] != 3 else bad[:1])
    cache.write(0, k, k)
    with pytest.raises(P.UfError):
        cache.attention(0, draw((5, 3, D), 0))
    for kw in (dict(tree=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(tree=torch.zeros(5, device="cuda")),
               dict(out=q.float()), dict(out=q[:4]), dict(lse=torch.empty((5, 2), device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            cache.attention(0, q, **kw)
    with pytest.raises(ValueError):
        cache.keep([0], [1], [2])
    with pytest.raises(ValueError):
        cache.keep([0], [1], [2], torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        cache.extend([0], [1], stream=0)
    with pytest.raises(ValueError):
        cache.keep([0], [1], [2], torch.zeros(2, dtype=torch.int32))


# ---- pages ---------------------------------------------------------------------------

def _values(ids, kv, layers):
    """K and V rows that name their token, layer, head and kind (bf16 holds integers up to 256)."""
    ids = torch.tensor(ids, dtype=torch.int64)
    col = torch.arange(D)
    out = []
    for layer in range(layers):
        h = torch.arange(kv)[None, :, None]
        base = torch.where(col[None, None, :] % 2 == 0, ids[:, None, None] % 251, ids[:, None, None] // 251 % 251)
        k = (base + col[None, None, :] // 64 + 2 * h + layer) % 256
        out.append((k.to(torch.bfloat16).cuda(), ((k + 17) % 256).to(torch.bfloat16).cuda()))
    return out


def _compare(cache, model, kv, layers):
    torch.cuda.synchronize()
    for s, rows in enumerate(model.rows):
        assert cache.pages(s) == model.table[s]
        if not rows:
            continue
        want = _values([r if r else 0 for r in rows], kv, layers)
        there = np.repeat(np.array(model.table[s]) >= 0, cache.desc.page_tokens)[:len(rows)]
        named = there & (np.array(rows) > 0)
        zero = there & (np.array(rows) == 0)
        for layer in range(layers):
            for got, w in zip(read(cache, s, layer), want[layer]):
                assert np.array_equal(got[named], f64(w)[named]), (s, layer)
                assert not got[zero].any()


@pytest.mark.parametrize("seed", range(4))
def test_pages_hold_what_the_model_says(seed):
    P = require_gpu()
    rng = np.random.default_rng(100 + seed)
    page, kv, layers, n_pages = (64, 128)[seed % 2], 1 + seed, 1 + seed % 3, 30
    cache, model = P.TokenCache(layers, kv, n_pages, 5, 900, page), O.PageModel(n_pages, 5, 900, page)
    poison(cache)
    next_id = 1
    for turn in range(60):
        what = rng.choice(["extend", "extend", "fork", "copy", "keep", "path", "trim", "free", "pack"])
        some = [int(s) for s in rng.permutation(5)[:rng.integers(1, 4)]]
        full, empty = [s for s in range(5) if model.rows[s]], [s for s in range(5) if not model.table[s]]
        if what == "extend":
            counts = [int(rng.choice([1, 2, 40, 130])) for _ in some]
            new = []
            for n in counts:
                new.append(list(range(next_id, next_id + n)))
                next_id += n
            if model.extend(some, new):
                cache.extend(some, counts)
                for layer, kv_rows in enumerate(_values(sum(new, []), kv, layers)):
                    cache.write(layer, *kv_rows)
        elif what == "fork" and full and empty:
            dst = empty[:int(rng.integers(1, 3))]
            model.fork([full[-1]] * len(dst), dst)
            cache.fork([full[-1]] * len(dst), dst)
        elif what == "copy" and full and empty:
            if model.copy([full[0]], [empty[0]]):
                cache.copy([full[0]], [empty[0]])
        elif what in ("keep", "path"):
            some = [s for s in some if -1 not in model.table[s] and model.rows[s]]
            starts = [int(rng.integers(0, len(model.rows[s]) + 1)) for s in some]
            index = []
            for s, a in zip(some, starts):
                n = len(model.rows[s])
                k = int(rng.integers(0, min(n - a, 16 if what == "path" else n) + 1))
                idx = np.sort(rng.permutation(np.arange(a, n))[:k]) if what == "path" else rng.integers(-2, n + 2, k)
                index.append([int(i) for i in idx])
            if some and model.keep(some, starts, index):
                flat = torch.tensor(sum(index, []), dtype=torch.int32, device="cuda")
                cache.keep(some, starts, [len(i) for i in index], flat)
        elif what == "trim" and rng.random() < 0.4:
            window, sinks = int(rng.integers(1, 300)), int(rng.integers(0, 100))
            model.trim(some, window, sinks)
            cache.trim(some, window, sinks)
        elif what == "free" and rng.random() < 0.4:
            model.free(some[:1])
            cache.free(some[:1])
        elif what == "pack":
            assert cache.pack() == model.pack()
        log(f"turn {turn} {what} {some}")
        _compare(cache, model, kv, layers)


def test_many_pages_in_one_call():
    """More words than a launch's arguments hold: extend, fork, copy, keep, trim, pack of 2,000 pages."""
    P = require_gpu()
    cache, model = P.TokenCache(1, 1, 9000, 4, 140000, 64), O.PageModel(9000, 4, 140000, 64)
    poison(cache)
    ids = list(range(1, 130001))
    for s, n in ((0, 130000), (1, 700)):
        assert model.extend([s], [ids[:n]])
        cache.extend([s], [n])
        cache.write(0, *_values(ids[:n], 1, 1)[0])
    _compare(cache, model, 1, 1)
    for what in ("fork", "copy"):
        getattr(model, what)([0], [2 if what == "fork" else 3])
        getattr(cache, what)([0], [2 if what == "fork" else 3])
    index = [list(range(1, 130000, 2)), list(range(0, 700, 3))]
    model.keep([2, 1], [0, 1], index)
    cache.keep([2, 1], [0, 1], [len(i) for i in index], torch.tensor(sum(index, []), dtype=torch.int32, device="cuda"))
    _compare(cache, model, 1, 1)
    model.trim([3], 1000, 70)
    cache.trim([3], 1000, 70)
    model.free([0])
    cache.free([0])
    assert cache.pack() == model.pack()
    _compare(cache, model, 1, 1)
    cache.extend([2], [1])
    model.extend([2], [[7]])
    cache.write(0, *_values([7], 1, 1)[0])
    q = draw((1, 1, D), 1, 0.001)
    out = cache.attention(0, q, lse=True)
    torch.cuda.synchronize()
    check_step(cache, 0, q, out, 0, 0, what="after all", seqs=[2], counts=[1])


def test_many_sequences_in_one_call():
    """More sequences than a launch's arguments hold words for."""
    P = require_gpu()
    n = 420
    cache, model = P.TokenCache(2, 1, 2600, 2 * n, 400, 64), O.PageModel(2600, 2 * n, 400, 64)
    poison(cache)
    rng = np.random.default_rng(1)
    ids, at = list(range(n)), 1
    for turn in range(2):
        new = []
        for _ in ids:
            k = int(rng.integers(1, 130)) if turn == 0 else 1
            new.append(list(range(at, at + k)))
            at += k
        assert model.extend(ids, new)
        cache.extend(ids, [len(x) for x in new])
        for layer, rows in enumerate(_values(sum(new, []), 1, 2)):
            cache.write(layer, *rows)
    q = draw((n, 3, D), 5, 0.01)
    out = cache.attention(1, q, 60, 1, lse=True)
    torch.cuda.synchronize()
    check_step(cache, 1, q, out, 60, 1, what="many", seqs=ids, counts=[1] * n)
    twins = [n + s for s in ids]
    model.fork(ids, twins)
    cache.fork(ids, twins)
    new = [[at + s] for s in ids]                         # every partly filled page is copied first
    assert model.extend(twins, new)
    cache.extend(twins, [1] * n)
    for layer, rows in enumerate(_values(sum(new, []), 1, 2)):
        cache.write(layer, *rows)
    _compare(cache, model, 1, 2)
    for most in (16, 100):                                # in place, and into fresh pages
        starts = [int(rng.integers(0, len(model.rows[s]) + 1)) for s in ids]
        index = [[int(x) for x in rng.integers(0, len(model.rows[s]), rng.integers(0, min(most, len(model.rows[s]) - a) + 1))]
                 for s, a in zip(ids, starts)]
        assert model.keep(ids, starts, index)
        cache.keep(ids, starts, [len(x) for x in index], torch.tensor(sum(index, []), dtype=torch.int32, device="cuda"))
        _compare(cache, model, 1, 2)
    model.free(twins)
    cache.free(twins)
    assert cache.pack() == model.pack()
    _compare(cache, model, 1, 2)


@pytest.mark.parametrize("kv,group,n,usual,others,held,window,sinks", [
    (2, 4, 150, 1, {70: 200, 140: 37}, 300, 0, 0),       # single tokens with two pieces of prompts, cut into slices
    (1, 3, 66, 1, {65: 500}, 20, 64, 5),
    (1, 40, 130, 0, {129: 4}, 150, 0, 0),                # tiles of one sequence at the end, the others do not grow
    (1, 2, 90, 17, {64: 1, 89: 3}, 2000, 0, 0),          # few rows beside many, over long ones
    (2, 1, 70, 20, {3: 700}, 65, 50, 2)])                # 33 rows and more only in one sequence
def test_steps_whose_sequences_grow_unequally(kv, group, n, usual, others, held, window, sinks):
    """A step of more than 64 sequences most of which bring other numbers of tokens than the longest, and a captured layer
    of such a step."""
    P = require_gpu()
    counts = [others.get(i, usual) for i in range(n)]
    lengths = [held if i in others or held < 1000 else 5 + i for i in range(n)]
    pages = sum(-(-(a + 4 * b) // 64) for a, b in zip(lengths, counts)) + 2
    cache = P.TokenCache(1, kv, pages, n, max(lengths) + 4 * max(counts), 64)
    poison(cache)
    seqs = [int(s) for s in np.random.default_rng(n).permutation(n)]
    fill(cache, seqs, lengths, 1)
    fill(cache, seqs, counts, 30)
    total = sum(counts)
    q = draw((total, kv * group, D), 7)
    log(f"unequal: kv={kv} group={group} n={n} usual={usual} others={others}")
    need = cache.work_bytes(kv * group, window, sinks)
    work = torch.full((need + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    out = cache.attention(0, q, window, sinks, lse=True, work=work[:need] if need else None)
    torch.cuda.synchronize()
    assert (work[need:] == 0x5A).all()
    check_step(cache, 0, q, out, window, sinks, what="unequal", seqs=seqs, counts=counts)

    k, v = draw((total, kv, D), 8), draw((total, kv, D), 9)
    o, lse = torch.empty_like(q), torch.empty((total, kv * group), device="cuda")
    cache.extend(seqs, counts)
    work = torch.empty(cache.work_bytes(kv * group, window, sinks) + 16, dtype=torch.uint8, device="cuda")

    def layer():
        cache.write(0, k, v)
        cache.attention(0, q, window, sinks, out=o, lse=lse, work=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for turn in range(3):
        order = list(seqs)
        if turn == 1:                                    # the same counts in the same places, other sequences
            same = [i for i in range(n) if i not in others]
            for i, j in zip(same, same[1:] + same[:1]):
                order[i] = seqs[j]
        if turn:
            cache.extend(order, counts)
        for t, seed in ((k, 10), (v, 11), (q, 12)):
            t.copy_(draw(t.shape, 100 * turn + seed))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_step(cache, 0, q, (o, lse), window, sinks, what=f"replay {turn}", seqs=order, counts=counts)


def test_a_speculative_run_equals_the_plain_one():
    """Prompt, draft trees, the accepted path kept, pages trimmed and packed: attention as of a sequence that
    holds only the accepted tokens, at every step."""
    P = require_gpu()
    kv, G, W, S = 2, 4, 150, 5
    cache = P.TokenCache(1, kv, 40, 3, 1000, 64)
    poison(cache)
    rng = np.random.default_rng(3)
    fill(cache, [0], [300], 1)
    cache.fork([0], [2])
    held = {0: read(cache, 0), 2: read(cache, 0)}
    for turn in range(12):
        widths = [int(rng.integers(1, 24)), int(rng.integers(1, 24))]
        cache.extend([0, 2], widths)
        k, v = draw((sum(widths), kv, D), 100 + turn), draw((sum(widths), kv, D), 200 + turn)
        cache.write(0, k, v)
        words, paths, at = [], [], 0
        for n in widths:
            own = []
            for t in range(n):
                parent = int(rng.integers(-1, t))
                own.append((own[parent] if parent >= 0 else 0) | 1 << t)
            words += own
            leaf = own[int(rng.integers(0, n))]
            paths.append([t for t in range(n) if leaf >> t & 1])
        q = draw((sum(widths), kv * G, D), 300 + turn)
        o = f64(cache.attention(0, q, W, S, tree=torch.tensor(words, dtype=torch.int64, device="cuda")))
        index, at = [], 0
        for s, n, path in zip((0, 2), widths, paths):
            kk, vv = held[s]
            rows = [at + t for t in path]
            held[s] = (np.concatenate([kk, f64(k)[rows]]), np.concatenate([vv, f64(v)[rows]]))
            see = O.sees(np.arange(len(kk), len(kk) + len(path)), np.arange(len(held[s][0])), W, S)
            check_rows(f64(q)[rows], o[rows], None, *held[s], see, what=f"turn {turn}")
            index += [len(kk) + t for t in path]
            at += n
        cache.keep([0, 2], [len(held[s][0]) - len(p) for s, p in zip((0, 2), paths)], [len(p) for p in paths],
                   torch.tensor(index, dtype=torch.int32, device="cuda"))
        cache.trim([0, 2], W, S)
        if turn % 4 == 3:
            cache.pack()
        for s in (0, 2):
            there = np.repeat(np.array(cache.pages(s)) >= 0, 64)[:cache.tokens(s)]
            assert cache.tokens(s) == len(held[s][0]) and not there.all() == (len(there) > 64 + 64 + W)
            for got, want in zip(read(cache, s), held[s]):
                assert np.array_equal(got[there], want[there])


def test_a_captured_layer_follows_the_steps():
    """write and attention captured once, replayed after later steps, between eager work and synchronisations."""
    P = require_gpu()
    cache = P.TokenCache(1, 2, 60, 2, 3000, 64)
    fill(cache, [0, 1], [1800, 90], 1)
    k, v, q = draw((2, 2, D), 2), draw((2, 2, D), 3), draw((2, 8, D), 4)
    cache.extend([0, 1], [1, 1])
    work = torch.empty(2 * cache.work_bytes(8, 1000, 4), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")

    def layer():
        cache.write(0, k, v)
        cache.attention(0, q, 1000, 4, out=o, lse=lse, work=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for turn in range(70):
        if turn:
            cache.extend([0, 1], [1, 1])
        if turn == 30:
            cache.trim([0, 1], 1000, 4)
        for t, seed in ((k, 10), (v, 11), (q, 12)):
            t.copy_(draw(t.shape, 100 * turn + seed))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        if turn % 10 in (0, 1, 9):
            check_step(cache, 0, q, (o, lse), 1000, 4, what=f"replay {turn}", seqs=[0, 1], counts=[1, 1])
            again = cache.attention(0, q, 1000, 4)
            torch.cuda.synchronize()
            assert torch.allclose(again.float(), o.float(), atol=2 ** -6)
