"""window_attention and its gradient on the GPU against the float64 oracle, within bounds that follow from their
roundings (oracle/tokens.py)."""

import math

import numpy as np
import pytest
import torch

from oracle import tokens as O
from tests.gpu_common import f64, log, require_gpu
from tests.test_gpu_tokens import D, SCALE, _only_those_that_see, check_rows, draw

pytestmark = pytest.mark.gpu

CASES = [
    # batch, tokens, kv heads, group, window, sinks, lengths
    (1, 1, 1, 1, 0, 0, None),
    (2, 65, 1, 1, 0, 0, None),
    (1, 200, 2, 3, 50, 4, None),                         # heads that do not divide a tile
    (2, 130, 1, 4, 1, 0, None),                          # a window of one token
    (1, 129, 1, 5, 0, 0, None),
    (3, 100, 2, 2, 33, 200, [100, 0, 37]),               # padding, an empty sequence, sinks past the end
    (2, 300, 1, 1, 64, 128, [1, 299]),
    (1, 1500, 1, 2, 20, 3, None),                        # the sinks' rows are cut into parts
    (2, 700, 1, 1, 17, 130, [700, 333]),                 # two tiles of sinks
    (1, 40, 1, 130, 7, 2, None),                         # a group larger than a tile
    (1, 700, 1, 1, 1 << 30, 1, None),                    # a window past every length
]


def run_all(P, q, k, v, do, window, sinks, lengths=None, scale=None):
    o, lse = P.window_attention(q, k, v, window, sinks, scale, lengths)
    return (o, lse) + tuple(P.window_attention_bwd(q, k, v, o, lse, do, window, sinks, scale, lengths))


def check_all(q, k, v, do, out, window, sinks, lengths=None, scale=SCALE):
    B, n, Hq, _ = q.shape
    G = Hq // k.shape[2]
    q, k, v, do = f64(q), f64(k), f64(v), f64(do)
    o, lse, dq, dk, dv = (f64(t) for t in out)
    worst = {}
    for b in range(B):
        L = n if lengths is None else lengths[b]
        for t in (o, dq, dk, dv):
            assert not t[b, L:].any()
        assert (lse[b, :, L:] == -np.inf).all()
        if L == 0:
            continue
        see = O.sees(np.arange(L), np.arange(L), window, sinks)
        check_rows(q[b, :L], o[b, :L], lse[b, :, :L].T, k[b, :L], v[b, :L], see, scale)
        for hk in range(k.shape[2]):
            parts = [O.grads(q[b, :L, h], k[b, :L, hk], v[b, :L, hk], do[b, :L, h], see, scale)
                     for h in range(hk * G, (hk + 1) * G)]
            for g, (part, h) in enumerate(zip(parts, range(hk * G, (hk + 1) * G))):
                want, bound = part[0]
                off = np.abs(dq[b, :L, h] - want) / bound
                assert (off <= 1).all(), ("dq", b, h, off.max())
                worst["dq"] = max(worst.get("dq", 0), off.max())
            for name, got, i in (("dk", dk, 1), ("dv", dv, 2)):
                want, bound = sum(p[i][0] for p in parts), sum(p[i][1] for p in parts)
                off = np.abs(got[b, :L, hk] - want) / bound
                assert (off <= 1).all(), (name, b, hk, off.max())
                worst[name] = max(worst.get(name, 0), off.max())
    log("  worst of the bounds: " + ", ".join(f"{k} {v:.3f}" for k, v in worst.items()))


@pytest.mark.parametrize("batch,tokens,kv,group,window,sinks,lengths", CASES)
def test_forward_and_backward(batch, tokens, kv, group, window, sinks, lengths):
    P = require_gpu()
    q, do = draw((batch, tokens, kv * group, D), 1, 1.25), draw((batch, tokens, kv * group, D), 4)
    k, v = draw((batch, tokens, kv, D), 2), draw((batch, tokens, kv, D), 3)
    lens = None
    if lengths is not None:                              # padding is never read
        lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lengths):
            for t in (q, k, v, do):
                t[b, n:] = float("nan")
    log(f"window batch={batch} tokens={tokens} kv={kv} group={group} window={window} sinks={sinks} lengths={lengths}")
    out = run_all(P, q, k, v, do, window, sinks, lens)
    torch.cuda.synchronize()
    check_all(*(torch.nan_to_num(t) for t in (q, k, v, do)), out, window, sinks, lengths)


def test_strided_views_of_one_projection_and_large_logits():
    P = require_gpu()
    B, n, Hq, Hk = 2, 333, 6, 2
    qkv = draw((B, n, Hq + 2 * Hk, D), 1)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    k[:, ::50] *= 20
    do = draw((B, n, Hq, D), 2)
    out = run_all(P, q, k, v, do, 90, 2, scale=0.2)
    torch.cuda.synchronize()
    check_all(q, k, v, do, out, 90, 2, scale=0.2)
    # heads outermost, and one row of keys for every batch
    kt, vt = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (k, v))
    for a, b in zip(out, run_all(P, q, kt, vt, do, 90, 2, scale=0.2)):
        assert torch.equal(a, b)
    shared = [t[:1].expand(B, -1, -1, -1) for t in (k, v)]
    out = run_all(P, q, *shared, do, 90, 2)
    torch.cuda.synchronize()
    check_all(q, *shared, do, out, 90, 2)


def test_more_than_two_to_the_31_elements():
    """Queries, outputs and their gradients past 32-bit offsets: the last tokens, as a sequence of their own."""
    P = require_gpu()
    n, Hq, Hk, W, m = 263_000, 64, 8, 40, 150
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, do = (torch.randn((1, n, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k, v = (torch.randn((1, n, Hk, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    assert q.numel() > 2 ** 31
    o, lse, dq, dk, dv = run_all(P, q, k, v, do, W, 0)
    tail = [t[:, -m - W:].contiguous() for t in (q, k, v, do)]
    want = run_all(P, *tail, W, 0)
    torch.cuda.synchronize()
    # a row's products are the same ones, in tiles that begin elsewhere: fp32 sums in another order, then one rounding
    for got, alone in ((o, want[0]), (dq, want[2])):
        assert (got[:, -m:].float() - alone[:, -m:].float()).abs().max() < 2 ** -5
    for got, alone in ((dk, want[3]), (dv, want[4])):
        a, b = got[:, -m:].float(), alone[:, -m:].float()
        assert (a - b).abs().max() < 2 ** -5 * b.abs().max()
    assert (lse[:, :, -m:] - want[1][:, :, -m:]).abs().max() < 1e-4
    check_all(*(t[:, :m] for t in (q, k, v, do)), run_all(P, *(t[:, :m].contiguous() for t in (q, k, v, do)), W, 0), W, 0)


def test_sinks_of_many_tiles():
    """Key tiles of sinks that fill the GPU by themselves are not cut; few of them are."""
    P = require_gpu()
    for tokens, kv, sinks in ((2600, 1, 2500), (2600, 8, 300)):
        q, do = draw((1, tokens, kv, D), 1), draw((1, tokens, kv, D), 2)
        k, v = draw((1, tokens, kv, D), 3), draw((1, tokens, kv, D), 4)
        out = run_all(P, q, k, v, do, 30, sinks)
        torch.cuda.synchronize()
        h = slice(kv - 1, kv)
        check_all(*(t[:, :, h] for t in (q, k, v, do)),
                  (out[0][:, :, h], out[1][:, h], out[2][:, :, h], out[3][:, :, h], out[4][:, :, h]), 30, sinks)


@pytest.mark.parametrize("kind", ["v inf", "v nan", "k nan"])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(kind):
    P = require_gpu()
    q, k, v = draw((1, 400, 6, D), 1), draw((1, 400, 2, D), 2), draw((1, 400, 2, D), 3)
    bad = [130, 131, 300]
    (k if kind[0] == "k" else v)[:, bad, 1] = float(kind[2:])
    o, lse = P.window_attention(q, k, v, 40, 5)
    torch.cuda.synchronize()
    see = O.sees(np.arange(400), np.arange(400), 40, 5)
    o, lse = f64(o)[0], f64(lse)[0].T
    check_rows(f64(q)[0, :, :3], o[:, :3], lse[:, :3], f64(k)[0, :, :1], f64(v)[0, :, :1], see)
    _only_those_that_see(f64(q)[0, :, 3:], o[:, 3:], lse[:, 3:], f64(k)[0, :, 1:], f64(v)[0, :, 1:], see, bad)


def test_padding_has_zero_gradients_beside_values_that_are_not_finite():
    P = require_gpu()
    lengths = torch.tensor([70, 200, 1], dtype=torch.int32, device="cuda")
    q, k, v, do = (draw((3, 300, h, D), i) for i, h in enumerate((6, 2, 2, 6)))
    for t in (k, v):
        t[:, [0, 60, 190]] = float("nan")
    o, lse = P.window_attention(q, k, v, 30, 3, lengths=lengths)
    grads = P.window_attention_bwd(q, k, v, o, lse, do, 30, 3, lengths=lengths)
    torch.cuda.synchronize()
    for g in (o, *grads):
        for b, n in enumerate((70, 200, 1)):
            assert not g[b, n:].any()
            assert g[b, :n].isnan().any()
    assert (lse.transpose(1, 2)[1, 200:] == -float("inf")).all()


def test_the_same_bits_again_on_another_stream_and_from_a_graph():
    P = require_gpu()
    q, do = draw((1, 700, 4, D), 1), draw((1, 700, 4, D), 2)
    k, v = draw((1, 700, 2, D), 3), draw((1, 700, 2, D), 4)
    want = run_all(P, q, k, v, do, 40, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, lse = P.window_attention(q, k, v, 40, 3, stream=side)
    got = (o, lse) + tuple(P.window_attention_bwd(q, k, v, o, lse, do, 40, 3, stream=side))
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run_all(P, q, k, v, do, 40, 3)
    for turn in range(4):
        for t in (q, k, v, do):
            t.copy_(draw(t.shape, 10 * turn + t.shape[2]))
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, run_all(P, q, k, v, do, 40, 3)):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_the_cache_and_the_whole_sequence_agree():
    """A prompt through the cache in pieces, and the same tokens at once."""
    P = require_gpu()
    q, k, v = draw((1, 777, 6, D), 1), draw((1, 777, 2, D), 2), draw((1, 777, 2, D), 3)
    o, lse = P.window_attention(q, k, v, 200, 5)
    cache = P.TokenCache(1, 2, 20, 1, 777, 64)
    at = 0
    for n in (300, 1, 5, 470, 1):
        cache.extend([0], [n])
        cache.write(0, k[0, at:at + n], v[0, at:at + n])
        got, gl = cache.attention(0, q[0, at:at + n], 200, 5, lse=True)
        torch.cuda.synchronize()
        # both are within a bf16 rounding and their weights' of the exact result
        assert (got.float() - o[0, at:at + n].float()).abs().max() < 2 ** -5
        assert (gl - lse[0, :, at:at + n].T).abs().max() < 1e-4
        at += n


def test_wrappers_refuse():
    P = require_gpu()
    q, k = draw((1, 9, 4, D), 1), draw((1, 9, 2, D), 2)
    o, lse = P.window_attention(q, k, k)
    for bad in (k[:, :8], k.float(), k.cpu(), k.expand(2, -1, -1, -1), k[..., :64], k.clone().requires_grad_()):
        with pytest.raises((ValueError, TypeError)):
            P.window_attention(q, k, bad)
    with pytest.raises(P.UfError):
        P.window_attention(q[:, :, :3], k, k)
    with pytest.raises(P.UfError):
        P.window_attention(q, k, k, window=-1)
    for kw in (dict(lengths=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(lengths=torch.zeros(1, device="cuda")),
               dict(out=q.float()), dict(lse=lse[:, :2])):
        with pytest.raises((ValueError, TypeError)):
            P.window_attention(q, k, k, **kw)
    for args in ((o[:, :8], lse, q), (o, lse[:, :3], q), (o, lse, k)):
        with pytest.raises((ValueError, TypeError)):
            P.window_attention_bwd(q, k, k, *args)
    with pytest.raises(ValueError):
        P.window_attention_bwd(q, k, k, o, lse, q, work=torch.empty(16, dtype=torch.uint8, device="cuda"))
