"""Plain float64 definitions of the state operators: linear attention with a decay, its gradients with bounds on what
rounding may change, and the selection of a beam search."""

import numpy as np

BF16 = 2.0 ** -8      # relative half step
FP32 = 2.0 ** -24


def walk(x, y, z, g, scale, first=None, back=False):
    """One sequence and head, token by token.  x, y, z [n, D], g the log decay, first [D, D] the matrix before the first token
    (back: behind the last one).  Returns (out [n, D], the matrix at the end).

    Forwards M = e^g M + y z^T and out = scale M^T x; backwards M = M + scale y z^T, out = M^T x, M = e^g M."""
    n, D = x.shape
    M = np.zeros((y.shape[1], z.shape[1])) if first is None else np.array(first, float)
    out, L = np.zeros((n, z.shape[1])), np.exp(g)
    for t in (range(n - 1, -1, -1) if back else range(n)):
        if back:
            M = M + scale * np.outer(y[t], z[t])
            out[t] = M.T @ x[t]
            M = L * M
        else:
            M = L * M + np.outer(y[t], z[t])
            out[t] = scale * M.T @ x[t]
    return out, M


def attend(q, k, v, g, scale, state=None):
    """q [n, Hq, D], k and v [n, Hk, D], g [Hk], state [Hk, D, D] or None: (o [n, Hq, D], final [Hk, D, D])."""
    G = q.shape[1] // k.shape[1]
    o, final = np.zeros(q.shape), np.zeros((k.shape[1], k.shape[2], k.shape[2]))
    for h in range(q.shape[1]):
        e = h // G
        o[:, h], final[e] = walk(q[:, h], k[:, e], v[:, e], g[e], scale, None if state is None else state[e])
    return o, final


def grads(q, k, v, do, g, scale, state=None, dfinal=None):
    """(dq, dk, dv, dstate)."""
    Hk = k.shape[1]
    G = q.shape[1] // Hk
    dq, dk, dv, ds = np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape), np.zeros((Hk,) + k.shape[2:] * 2)
    for h in range(q.shape[1]):
        e = h // G
        # what the key head has from the final state counts once
        last = dfinal[e] if dfinal is not None and h % G == 0 else None
        dq[:, h] = walk(do[:, h], v[:, e], k[:, e], g[e], scale, None if state is None else state[e].T)[0]
        dk[:, e] += walk(v[:, e], do[:, h], q[:, h], g[e], scale, None if last is None else last.T, back=True)[0]
        dvh, dsh = walk(k[:, e], q[:, h], do[:, h], g[e], scale, last, back=True)
        dv[:, e] += dvh
        ds[e] += dsh
    return dq, dk, dv, ds


def steps(n, D=128):
    """fp32 roundings that a term passes on its way through n tokens, times a half step: the products' sums over D and over a
    chunk's tokens, the state's sums over all tokens, one factor and the parts' join a chunk, the weights, the scale.  Matrix
    cores may cut off where others round: a whole step each."""
    return 2 * FP32 * (n + n / 32 * 3 + 2 * D + 64)


def bf16_bound(exact, size, n, parts=2.0 ** -15):
    """Elementwise bound on a bf16 result off its exact value.  P, M and what is added to M go into products as two parts (or
    three) of 8 bits, the first cut off, the second rounded: 2^-7 2^-8 of what is left at most, each; then the result's own
    rounding."""
    a = size * (3 * parts + steps(n))
    return a + (np.abs(exact) + a) * BF16 + 1e-30


def fp32_bound(size, n):
    """The same of a state: what is added to it comes in three parts, 2^-7 2^-7 2^-8."""
    return size * (2.0 ** -22 + steps(n)) + 1e-37


def round_bf16(x):
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


# ---- selection ----------------------------------------------------------------------

def candidates(logits, scores, done=None, end=None, wide=np.float32):
    """One request: scores of all continuations, [beams, vocab], NaN where there is none.  logits float32 [beams, vocab]."""
    W, V = logits.shape
    out = np.full((W, V), np.nan, wide)
    with np.errstate(all="ignore"):
        for w in range(W):
            s = wide(scores[w])
            if done is not None and done[w]:
                out[w, end] = s
            else:
                x = logits[w].astype(np.float64)
                top = x.max() if np.isfinite(x.max()) else 0.0
                lse = wide(top + np.log(np.exp(x - top).sum()))
                out[w] = s + (logits[w].astype(wide) - lse)
    return np.where(out > -np.inf, out, np.nan).astype(wide)


def select(logits, scores, k, done=None, end=None):
    """(scores, parents, tokens) of the k best, equal scores by the lowest (beam, token)."""
    c = candidates(logits, scores, done, end)
    flat = c.reshape(-1)
    there = np.flatnonzero(~np.isnan(flat))
    best = there[np.lexsort((there, -flat[there]))][:k]
    pad = k - len(best)
    return (np.concatenate([flat[best], np.full(pad, -np.inf, np.float32)]),
            np.concatenate([best // c.shape[1], np.full(pad, -1)]), np.concatenate([best % c.shape[1], np.full(pad, -1)]))
