"""The token operators' results as norms over a tensor, on the GPU: no further from float64 than the stated roundings put
them (oracle/tokens.py; what that rejects is shown in test_oracle_token_norms.py)."""

import numpy as np
import pytest
import torch

from oracle import tokens as O
from tests.gpu_common import f64, log, require_gpu
from tests.test_gpu_tokens import D, SCALE, draw, fill, poison, read

pytestmark = pytest.mark.gpu


def held_to(name, got, before, *parts):
    off, limit = np.linalg.norm(got - before), O.norm_limit(before, *parts)
    size = np.linalg.norm(before)
    log(f"  {name}: off {off / size:.2e}, at most {limit / size:.2e}")
    assert off <= limit, name


@pytest.mark.parametrize("tokens,kv,group,window,sinks,length", [
    (300, 2, 1, 0, 0, 300), (300, 1, 3, 50, 4, 300), (400, 1, 2, 6, 2, 333), (700, 2, 1, 128, 130, 700), (1500, 1, 2, 20, 3, 1500),
    (2000, 1, 1, 1000, 0, 2000), (150, 1, 70, 40, 0, 150), (400, 3, 1, 3, 0, 400),
    (500, 1, 3, 120, 8, 500), (500, 1, 2, 100, 29, 500)])
def test_whole_sequences(tokens, kv, group, window, sinks, length):
    P = require_gpu()
    q, do = draw((1, tokens, kv * group, D), 1, 1.25), draw((1, tokens, kv * group, D), 2)
    k, v = draw((1, tokens, kv, D), 3), draw((1, tokens, kv, D), 4)
    lengths = None if length == tokens else torch.tensor([length], dtype=torch.int32, device="cuda")
    log(f"tokens={tokens} kv={kv} group={group} window={window} sinks={sinks} length={length}")
    out = P.window_attention(q, k, v, window, sinks, lengths=lengths)
    grads = P.window_attention_bwd(q, k, v, *out, do, window, sinks, lengths=lengths)
    torch.cuda.synchronize()
    n, H = length, kv * group
    q, k, v, do, o, dq, dk, dv = (f64(t)[0, :n] for t in (q, k, v, do, out[0], *grads))
    lse = f64(out[1])[0, :, :n]
    see = O.sees(np.arange(n), np.arange(n), window, sinks)
    want = {x: np.zeros_like(y) for x, y in (("o", o), ("round", o), ("dq", dq), ("dk", dk), ("dv", dv))}
    for h in range(H):
        one = q[:, h], k[:, h // group], v[:, h // group]
        before, want["o"][:, h] = O.rounded_attend(*one, see, SCALE)
        want["round"][:, h] = before - want["o"][:, h]
        g = O.rounded_grads(*one, do[:, h], o[:, h], lse[h], see, SCALE, O.few_keys(n, window, sinks, group, h % group))
        want["dq"][:, h] = g[0]
        want["dk"][:, h // group] += g[1]
        want["dv"][:, h // group] += g[2]
    held_to("o", o, want["o"], want["round"])
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        held_to(name, got, want[name])


@pytest.mark.parametrize("held,new,kv,group,window,sinks,split", [
    (3000, 1, 2, 8, 0, 0, True), (3000, 1, 2, 8, 0, 0, False), (500, 4, 4, 4, 100, 3, True), (20000, 1, 1, 16, 0, 0, True),
    (2000, 40, 1, 4, 0, 0, True), (900, 200, 2, 2, 300, 5, True), (0, 500, 1, 2, 0, 0, False)])
def test_over_the_cache(held, new, kv, group, window, sinks, split):
    P = require_gpu()
    cache = P.TokenCache(1, kv, (held + new) // 64 + 3, 1, held + new, 64)
    poison(cache)
    fill(cache, [0], [held], 1)
    fill(cache, [0], [new], 5)
    q = draw((new, kv * group, D), 9, 1.25)
    cache.n_cu = cache.n_cu if split else 0
    log(f"{held}+{new} kv={kv} group={group} window={window} sinks={sinks} split={split}")
    o, lse = cache.attention(0, q, window, sinks, lse=True)
    torch.cuda.synchronize()
    (k, v), q, o, lse = read(cache, 0), f64(q), f64(o), f64(lse)
    see = O.sees(np.arange(held, held + new), np.arange(held + new), window, sinks)
    want, rounds = np.zeros_like(o), np.zeros_like(o)
    for h in range(kv * group):
        one = q[:, h], k[:, h // group], v[:, h // group]
        before, want[:, h] = O.rounded_attend(*one, see, SCALE)
        rounds[:, h] = before - want[:, h]
        # LSE: scores in fp32 (8 sums of 16 products, 2^-24 of scores up to 16 before the scale each), weights below 1 with
        # an error of 2^-24 of their sum for each doubling of the keys, log2 and the product with ln 2
        assert np.abs(lse[:, h] - O.attend(*one, see, SCALE)[1]).max() < 2e-5
    held_to("o", o, want, rounds)
