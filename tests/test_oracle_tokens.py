"""The token operators' oracle against facts outside itself, and the token cache's page tables (dry runs,
no GPU) against the oracle's model, with every refusal that the host can force."""

import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from oracle import tokens as O


@pytest.fixture(scope="module")
def P():
    import paper_2606_09150_amd as pkg
    pkg.load()
    return pkg


# ---- the oracle -------------------------------------------------------------------

@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 0), (3, 2), (2, 5), (50, 4)])
def test_visibility_by_loops(window, sinks):
    see = O.sees(np.arange(9), np.arange(9), window, sinks)
    for i in range(9):
        want = {j for j in range(9) if j <= i and (window == 0 or i - j < window or j < sinks)}
        assert set(np.flatnonzero(see[i])) == want


def test_a_tree_node_sees_what_its_path_alone_would():
    # root 0, its children 1 and 2, node 3 below 2
    bits = [0b0001, 0b0011, 0b0101, 0b1101]
    paths = [[0], [0, 1], [0, 2], [0, 2, 3]]
    for window, sinks in ((0, 0), (4, 0), (5, 2)):
        see = O.tree_sees(6, bits, window, sinks)
        for t, path in enumerate(paths):
            alone = O.sees([6 + len(path) - 1], np.arange(6 + len(path)), window, sinks)[0]
            assert list(see[t, :6]) == list(alone[:6])
            assert set(np.flatnonzero(see[t, 6:])) == set(path) and alone[6:].all()
    assert not O.tree_sees(0, [0, 1]) [0].any()


def test_attention_matches_torch_and_its_gradients_match_differences():
    rng = np.random.default_rng(0)
    n, m, d = 5, 7, 6
    q, k, v, do = (rng.standard_normal(s) for s in ((n, d), (m, d), (m, d), (n, d)))
    see = O.sees(np.arange(2, 7), np.arange(7), 3, 1)
    see[1] = False                                     # a row that sees nothing
    o, lse, _ = O.attend(q, k, v, see, 0.3)
    rows = [0, 2, 3, 4]
    want = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(x)[None] for x in (q, k, v)), attn_mask=torch.from_numpy(see)[None], scale=0.3)[0].numpy()
    assert np.allclose(o[rows], want[rows], atol=1e-12) and not o[1].any() and lse[1] == -np.inf
    got = [g for g, _ in O.grads(q, k, v, do, see, 0.3)]
    for x, g in zip((q, k, v), got):
        for at in [(0, 0), (1, 3), (3, 5), (4, 2)]:
            keep, h = x[at], 1e-6
            x[at] = keep + h
            up = (O.attend(q, k, v, see, 0.3)[0] * do).sum()
            x[at] = keep - h
            down = (O.attend(q, k, v, see, 0.3)[0] * do).sum()
            x[at] = keep
            assert abs((up - down) / (2 * h) - g[at]) < 1e-8


# ---- page tables ------------------------------------------------------------------

def _dry(P, n_pages=40, max_seqs=6, max_tokens=700, page=64, layers=2, kv_heads=3):
    return P.TokenCache(layers, kv_heads, n_pages, max_seqs, max_tokens, page, flags=P._lib.UF_F_DRYRUN)


def _same(cache, model):
    for s, (pages, rows) in enumerate(zip(model.table, model.rows)):
        assert cache.pages(s) == pages and cache.tokens(s) == len(rows)
    assert cache.info().free_pages == model.free_pages()


def _call(P, f):
    try:
        f()
        return True
    except P.UfError as e:
        assert e.status == P._lib.UF_ERR_CAPACITY, e
        return False


@pytest.mark.parametrize("seed", range(8))
def test_pages_match_the_model_under_random_calls(P, seed):
    rng = np.random.default_rng(seed)
    page = (64, 128)[seed % 2]
    cache, model = _dry(P, n_pages=int(rng.integers(6, 40)), page=page), None
    model = O.PageModel(cache.desc.n_pages, 6, 700, page)
    refused = 0
    for _ in range(150):
        what = rng.choice(["extend", "extend", "extend", "fork", "copy", "keep", "cut", "trim", "free", "pack"])
        some = [int(s) for s in rng.permutation(6)[:rng.integers(1, 4)]]
        full = [s for s in range(6) if model.rows[s]]
        empty = [s for s in range(6) if not model.table[s]]
        if what == "extend":
            counts = [int(rng.choice([0, 1, 5, 64, 150])) for _ in some]
            done = model.extend(some, [[0] * n for n in counts])
            assert _call(P, lambda: cache.extend(some, counts)) == done
            refused += not done
            if done:
                info = cache.info()
                assert (info.step_seqs, info.step_tokens, info.step_longest) == (len(some), sum(counts), max(counts))
        elif what in ("fork", "copy") and full and empty:
            src, dst = [full[0]] * len(empty[:2]), empty[:2]
            done = model.fork(src, dst) is None if what == "fork" else model.copy(src, dst)
            assert _call(P, lambda: getattr(cache, what)(src, dst)) == done
        elif what in ("keep", "cut"):
            some = [s for s in some if -1 not in model.table[s]]
            starts = [int(rng.integers(0, len(model.rows[s]) + 1)) for s in some]
            room = [len(model.rows[s]) - a for s, a in zip(some, starts)]
            counts = [0 if what == "cut" else int(rng.integers(0, n + 1)) for n in room]
            if some:
                done = model.keep(some, starts, [[a] * n for a, n in zip(starts, counts)])
                assert _call(P, lambda: cache.keep(some, starts, counts, np.zeros(1))) == done
        elif what == "trim":
            window, sinks = int(rng.integers(1, 300)), int(rng.integers(0, 200))
            model.trim(some, window, sinks)
            cache.trim(some, window, sinks)
        elif what == "free" and rng.random() < 0.5:
            model.free(some)
            cache.free(some)
        elif what == "pack":
            assert cache.pack() == model.pack()
        _same(cache, model)
    assert refused or cache.desc.n_pages > 20


def test_branches_of_a_partly_filled_page(P):
    c = _dry(P)
    c.extend([0], [70])
    c.fork([0, 0], [1, 2])
    assert c.pages(1) == c.pages(2) == [0, 1] and c.info().free_pages == 38
    c.extend([1, 2, 0], [1, 1, 1])                     # the last of the three keeps the shared page
    assert [c.pages(s) for s in (0, 1, 2)] == [[0, 1], [0, 2], [0, 3]]
    c.free([0])
    c.extend([3], [10])
    assert c.pages(3) == [1]                           # page 0 still has users
    full = _dry(P, n_pages=2)
    full.extend([0], [100])
    full.fork([0], [1])
    with pytest.raises(P.UfError) as e:
        full.extend([0], [1])                          # no page to copy into
    assert e.value.status == P._lib.UF_ERR_CAPACITY and full.tokens(0) == 100 and full.pages(0) == [0, 1]


def test_a_step_ends_when_its_sequences_are_cut_or_freed(P):
    c = _dry(P)
    c.extend([0, 1], [5, 6])
    c.fork([0], [2])
    c.trim([0, 1], 3)
    c.pack()
    assert c.info().step_seqs == 2
    c.keep([2], [1], [0])
    assert c.info().step_seqs == 2
    c.keep([1], [6], [0])
    assert c.info().step_seqs == 0
    for call in (lambda: c.write(0, None, None), lambda: c.attention(0, 6)):
        with pytest.raises(P.UfError) as e:
            call()
        assert e.value.status == P._lib.UF_ERR_EMPTY
    c.extend([1], [1])
    c.free([1])
    assert c.info().step_seqs == 0


def test_refusals(P):
    L, T = P._lib, P._tokens
    ARG, UNSUP, CAP, EMPTY = L.UF_ERR_ARG, L.UF_ERR_UNSUPPORTED, L.UF_ERR_CAPACITY, L.UF_ERR_EMPTY

    def status(f):
        with pytest.raises(P.UfError) as e:
            f()
        assert len(str(e.value).split(": ", 2)[-1]) > 5           # the text of uf_last_error
        return e.value.status

    for bad, want in ((dict(layers=0), ARG), (dict(kv_heads=0), ARG), (dict(n_pages=0), ARG), (dict(max_seqs=0), ARG),
                      (dict(max_tokens=0), ARG), (dict(page=0), ARG), (dict(page=32), UNSUP), (dict(max_seqs=65536), ARG),
                      (dict(max_seqs=60000, max_tokens=1 << 30), ARG)):
        assert status(lambda: _dry(P, **bad)) == want, bad
    assert status(lambda: P.TokenCache(1, 1, 1, 1, 1, head_dim=64, flags=1)) == UNSUP
    assert status(lambda: P.TokenCache(1, 1, 1, 1, 1, flags=3)) == ARG
    desc = T.uft_desc(1, 1, 128, 64, 4, 2, 100, 0)
    assert status(lambda: T.uft_create(desc, None, None)) == ARG
    c = _dry(P)
    c.extend([0], [100])
    before = (c.pages(0), c.info().free_pages, c.info().step_tokens)
    for f in (lambda: c.extend([], []), lambda: c.extend([6], [1]), lambda: c.extend([-1], [1]), lambda: c.extend([1, 1], [1, 1]),
              lambda: c.extend([1], [-1]), lambda: c.fork([0], [0]), lambda: c.fork([0, 0], [1, 1]), lambda: c.fork([9], [1]),
              lambda: c.keep([0], [101], [0]), lambda: c.keep([0], [-1], [0]), lambda: c.keep([0], [50], [51], 1),
              lambda: c.keep([0, 0], [1, 1], [0, 0]), lambda: c.trim([0], 0), lambda: c.trim([0], 1, -1), lambda: c.free([7]),
              lambda: c.attention(2, 3), lambda: c.attention(-1, 3), lambda: c.attention(0, 4), lambda: c.attention(0, 0),
              lambda: c.attention(0, 3, -1), lambda: c.attention(0, 3, 1, -1), lambda: c.attention(0, 3, scale=0.0),
              lambda: c.attention(0, 3, scale=math.inf), lambda: c.attention(0, 3, scale=1e-39),
              lambda: c.write(2, None, None), lambda: c.tokens(6), lambda: c.pages(-1)):
        assert status(f) == ARG
    assert status(lambda: c.fork([1], [2])) == EMPTY
    assert status(lambda: c.copy([1], [2])) == EMPTY
    assert status(lambda: c.extend([0], [601])) == CAP
    assert status(lambda: c.extend([1, 2, 3, 4], [700] * 4)) == CAP
    assert (c.pages(0), c.info().free_pages, c.info().step_tokens) == before
    c.trim([0], 1)
    assert c.pages(0) == [-1, 1]
    assert status(lambda: c.keep([0], [10], [0])) == ARG              # its page has gone
    c.keep([0], [70], [0])
    c.extend([0], [65])
    node = torch.zeros(1, dtype=torch.int64)
    assert status(lambda: c.attention(0, 3, tree=node)) == UNSUP         # 65 nodes
    c.extend([0], [9])
    assert status(lambda: c.attention(0, 3, 8, tree=node)) == ARG        # a window smaller than the tree
    with pytest.raises(ValueError):
        c.extend([0, 1], [1])
    with pytest.raises(ValueError):
        c.keep([0], [1], [2])
    with pytest.raises(TypeError):
        c.extend(torch.zeros(1), [1])
    null = T.uft_stride(0, 0, 0)
    w = lambda **kw: T.uft_window_desc(**dict(dict(batch=1, tokens=5, q_heads=4, kv_heads=2, head_dim=128, window=0, sinks=0,  # noqa: E731
                                                   scale=0.1, q=null, k=null, v=null), **kw))
    for bad, want in ((dict(batch=0), ARG), (dict(tokens=0), ARG), (dict(q_heads=3), ARG), (dict(kv_heads=0), ARG),
                      (dict(head_dim=64), UNSUP), (dict(window=-1), ARG), (dict(sinks=-1), ARG), (dict(scale=-1.0), ARG),
                      (dict(scale=math.nan), ARG), (dict(q=T.uft_stride(0, 4, 8)), ARG), (dict(k=T.uft_stride(0, -8, 8)), ARG),
                      (dict(v=T.uft_stride(0, (1 << 24) + 8, 8)), ARG), (dict(tokens=(1 << 30) + 1), ARG),
                      (dict(batch=1 << 20, tokens=1 << 20), ARG)):
        assert status(lambda: T.uft_window_bwd_work_bytes(w(**bad))) == want, bad
    assert status(lambda: T.uft_window_fwd(w(), None, None, None, None, None, None)) == ARG
    assert status(lambda: T.uft_window_bwd(w(), *[None] * 11)) == ARG


@pytest.mark.parametrize("held,new,one,one_held", [(4000, 1, 512, 4000), (10, 16, 1, 100000), (900, 1, 700, 0), (300, 9, 8, 5000)])
def test_scratch_follows_the_sequences_that_are_cut(P, held, new, one, one_held):
    """A sequence beside 200 others that bring other numbers of rows: the step's scratch is at most twice that of the two
    kinds in steps of their own."""
    c = _dry(P, 60000, 201, 200000, kv_heads=8)
    c.n_cu = 256
    c.extend(list(range(201)), [one_held] + [held] * 200)
    need = []
    for seqs, counts in (([0], [one]), (list(range(1, 201)), [new] * 200), (list(range(201)), [one] + [new] * 200)):
        c.extend(seqs, counts)
        need.append(c.work_bytes(32))
        c.keep(seqs, [c.tokens(s) - n for s, n in zip(seqs, counts)], [0] * len(seqs))
    assert need[2] <= 2 * (need[0] + need[1]), need


def test_integers_that_32_bits_cannot_hold(P):
    c = _dry(P)
    c.extend([0], [5])
    for f in (lambda: c.attention(0, 3, 2 ** 32), lambda: c.attention(2 ** 32, 3), lambda: c.attention(0, 3, 1, 2 ** 31),
              lambda: c.trim([0], 2 ** 32 + 1), lambda: c.write(2 ** 32, None, None), lambda: c.tokens(2 ** 32),
              lambda: _dry(P, max_tokens=2 ** 32 + 5), lambda: c.work_bytes(3, 2 ** 33)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(OverflowError):
        c.extend([0], [2 ** 32])
    with pytest.raises(TypeError):
        c.attention(0, 3, 1.5)
    assert c.tokens(np.int64(0)) == 5
    c.attention(np.int64(0), 3, np.int32(4))


def test_library_exports_every_declared_symbol(P):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = sorted(set(re.findall(r"^\s*int\s+(uft_\w+)\s*\(", open(os.path.join(root, "include", "uft.h")).read(), re.M)))
    out = subprocess.run(["nm", "-D", "--defined-only", P._lib.LIB_PATH], capture_output=True, text=True).stdout
    assert len(names) == 20 and sorted(set(re.findall(r"\sT\s(uft_\w+)$", out, re.M))) == names
    assert set(P._tokens._SIGNATURES) == set(names)


def test_the_header_is_plain_c(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "a.c"
    src.write_text('#include "uft.h"\nint main(void) { uft_window_desc d = {0}; return (int)d.batch; }\n')
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-pedantic", f"-I{root}/include", "-fsyntax-only", str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_wrappers_refuse_host_tensors(P):
    x = torch.zeros((1, 5, 2, 128), dtype=torch.bfloat16)
    for q, k, error in ((x, x, ValueError), (x.float(), x, TypeError), (x[0], x, ValueError), (None, x, ValueError)):
        with pytest.raises(error):
            P.window_attention(q, k, k)
