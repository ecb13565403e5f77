"""Plain float64 definitions of the token operators: which keys a query sees, attention and
its gradients with bounds on what rounding may change, and the token cache's pages."""

import numpy as np

BF16 = 2.0 ** -8      # relative half step
FP16 = 2.0 ** -11
FP32 = 2.0 ** -24


def sees(pos, keys, window=0, sinks=0):
    """bool [queries, keys] from their positions."""
    i, j = np.asarray(pos)[:, None], np.asarray(keys)[None, :]
    near = (i - j < window) | (j < sinks) if window else np.ones((i.shape[0], j.shape[1]), bool)
    return (j <= i) & near


def tree_sees(held, bits, window=0, sinks=0):
    """bool [nodes, held + nodes]: ``bits`` are the nodes that each node sees, as integers."""
    n = len(bits)
    node = np.array([[(int(b) >> t) & 1 for t in range(n)] for b in bits], bool).reshape(n, n)
    pos = held + np.maximum(node.sum(1) - 1, 0)
    return np.concatenate([sees(pos, np.arange(held), window, sinks), node], axis=1)


def attend(q, k, v, see, scale):
    """One sequence and head: q [n, D], k and v [m, D], see [n, m].  Returns o, lse, p."""
    s = (q @ k.T) * scale
    top = np.where(see, s, -np.inf).max(axis=1, initial=-np.inf)
    e = np.where(see, np.exp(np.where(see, s, -np.inf) - np.where(np.isfinite(top), top, 0.0)[:, None]), 0.0)
    total = e.sum(1)
    p = e / np.where(total > 0, total, 1.0)[:, None]
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, np.log(total) + np.where(np.isfinite(top), top, 0.0), -np.inf)
    return p @ v, lse, p


def score_error(q, k, scale):
    """What fp32 products and sums may change a score by: D products and sums, the scale, exp2's argument."""
    size = float((np.abs(q) @ np.abs(k).T).max()) * scale
    return (q.shape[1] + 8) * FP32 * max(size, 1.0)


def attend_bound(q, k, v, p, o, scale):
    """Elementwise bound on |O - exact|: each weight is off by a bf16 half step and by what its score is (twice, with
    the sum's); sums over the keys in fp32; one rounding of O to bf16."""
    weight = BF16 + 2 * score_error(q, k, scale) + (2 * k.shape[0] + 64) * FP32
    a = (p @ np.abs(v)) * weight
    return a + (np.abs(o) + a) * BF16 + 1e-30


def lse_bound(q, k, lse, scale):
    return score_error(q, k, scale) + (k.shape[0] + 64) * FP32 + 8 * FP32 * (1 + np.where(np.isfinite(lse), np.abs(lse), 0))


def grads(q, k, v, do, see, scale):
    """(dq, dk, dv) of one head and their bounds."""
    o, _, p = attend(q, k, v, see, scale)
    delta = (do * o).sum(1, keepdims=True)
    dp = do @ v.T
    ds = p * (dp - delta)
    dq, dk, dv = scale * ds @ k, scale * ds.T @ q, p.T @ do
    # P is off as its score is.  For dV it is rounded to bf16; for dQ it stays fp32, and dS formed from it is rounded to two
    # bf16 parts (the second a half step off the remainder, which is a half step of dS); for dK it passes through fp16,
    # 2^15 times as large: off by 2^-11, or where that is subnormal (spacing 2^-24, weights below 2^-14 / 2^15) by half a
    # spacing, 2^-25 / 2^15, whatever its own size; and dS is rounded once.  For dQ delta comes from O rounded to bf16, whose
    # own error is attend_bound's (where rows see few keys it is corrected as for dK: the bound is wide there); for dK
    # it is the sum of P dP over the row's keys.  Sums in fp32; one rounding of each result to bf16
    off = 2 * score_error(q, k, scale) + (2 * max(k.shape[0], q.shape[0]) + 64) * FP32
    d_delta = (np.abs(do) * attend_bound(q, k, v, p, o, scale)).sum(1, keepdims=True)
    d_dp = (np.abs(do) @ np.abs(v).T + np.abs(delta)) * (do.shape[1] + 8) * FP32
    e_q = np.abs(ds) * off + p * (d_delta + d_dp) * (1 + off)     # what P and dP - delta are off by
    e_q += (np.abs(ds) + e_q) * BF16 ** 2
    d_sum = (p * (np.abs(dp) * off + d_dp)).sum(1, keepdims=True) + np.abs(delta) * off
    e_k = np.abs(ds) * (off + FP16) + (p * (1 + off + FP16) + 2.0 ** -40 * see) * (d_sum + d_dp) + 2.0 ** -40 * np.abs(dp - delta) * see
    e_k += (np.abs(ds) + e_k) * BF16
    e_p = p * (off + BF16 * (1 + off))
    b_dq, b_dk, b_dv = scale * e_q @ np.abs(k), scale * e_k.T @ np.abs(q), e_p.T @ np.abs(do)
    sums = (2 * max(k.shape[0], q.shape[0]) + 64) * FP32
    return [(g, b + s * sums + (np.abs(g) + b) * BF16 + 1e-30)
            for g, b, s in ((dq, b_dq, scale * np.abs(ds) @ np.abs(k)), (dk, b_dk, scale * np.abs(ds).T @ np.abs(q)),
                            (dv, b_dv, p.T @ np.abs(do)))]


# ---- what the stated roundings alone do, as norms ---------------------------------
#
# The bounds above add absolute values: they hold for every element, and leave room for a rounding too many.  Norms over a
# tensor leave none: the same operations with exactly the stated roundings, everything else in float64.

def keep_bits(x, bits):
    """x to so many significant bits, ties to even (bf16: 8)."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def rounded_attend(q, k, v, see, scale, p_bits=8):
    """(O before its own rounding, O exactly): weights rounded for their product with V.  They are formed relative to an
    offset that need not be the row's largest score (it is raised on a row's first units only, and by far larger scores
    later), so the largest is off as the others are: here relative to the sum, where none is a power of two by design."""
    o, _, p = attend(q, k, v, see, scale)
    return keep_bits(p, p_bits) @ v, o


def few_keys(n, window=0, sinks=0, group=1, g=0):
    """bool [n]: the tokens whose rows, of head g of a group, lie in tiles of 128 rows that see 128 keys at most."""
    row = np.arange(n) * group + g
    last = (np.minimum(row // 128 * 128 + 128, n * group) - 1) // group
    return np.minimum(last + 1, window + sinks if window else n) <= 128


def rounded_grads(q, k, v, do, o, lse, see, scale, few, p_bits=8, ds_bits=(16, 8), delta_off=0.0, ds_off=0.0):
    """dq, dk, dv of one head before their own rounding, from O and LSE as the forward left them.  ds_bits: of dS for dQ
    (two parts of 8) and for dK.  delta: the sum of P dP for dK and for dQ's rows of ``few`` keys, for its others from O."""
    s = np.where(see, q @ k.T * scale, -np.inf)
    with np.errstate(invalid="ignore"):
        p = np.where(see, np.exp(s - np.where(np.isfinite(lse), lse, 0.0)[:, None]), 0.0)
    dp = do @ v.T
    exact = (p * dp).sum(1, keepdims=True)
    delta = np.where(few[:, None], exact, (do * o).sum(1, keepdims=True))
    hand = (p * 2.0 ** 15).astype(np.float16).astype(np.float64) * 2.0 ** -15
    dsq, dsk = (keep_bits(x * (dp - d * (1 + delta_off)) * (1 + ds_off), b) for x, d, b in zip((p, hand), (delta, exact), ds_bits))
    return scale * dsq @ k, scale * dsk.T @ q, keep_bits(p, p_bits).T @ do


def norm_limit(before, *parts):
    """The most that a result may be off, as a norm: its own rounding to bf16, ``parts`` and 2^-11 of the result for fp32, all
    independent of each other, and a tenth more of their squares for chance.  Where fp32 (scores and LSE off by e, 1e-6 at
    scores of 10) carries a value over a rounding's border it changes by a step u, with chance e / u: sqrt(e u) of a weight,
    7e-5 at u = 2^-8, and sums in fp32 are off by less."""
    own = [keep_bits(before, 8) - before, 2.0 ** -11 * before, *parts]
    return np.sqrt(1.1 * sum(float((x * x).sum()) for x in own))


class PageModel:
    """Pages of a token cache, and which token (any value) lies where."""

    IN_PLACE = 16

    def __init__(self, n_pages, max_seqs, max_tokens, page):
        self.T, self.n_pages, self.max_tokens = page, n_pages, max_tokens
        self.uses = [0] * n_pages
        self.table = [[] for _ in range(max_seqs)]
        self.rows = [[] for _ in range(max_seqs)]      # the token at each position (None: no value)

    def free_pages(self):
        return self.uses.count(0)

    def take(self):
        p = self.uses.index(0)
        self.uses[p] = 1
        return p

    def drop(self, pages):
        for p in pages:
            if p >= 0:
                self.uses[p] -= 1

    def extend(self, seqs, tokens):
        """tokens[i]: the values that sequence seqs[i] grows by.  False (and nothing done) where pages do not suffice."""
        before = (list(self.uses), [list(t) for t in self.table])
        try:
            for s, new in zip(seqs, tokens):
                if len(self.rows[s]) + len(new) > self.max_tokens:
                    raise ValueError
                if new and len(self.rows[s]) % self.T and self.uses[self.table[s][-1]] > 1:
                    old = self.table[s][-1]
                    self.table[s][-1] = self.take()
                    self.uses[old] -= 1
                while len(self.table[s]) * self.T < len(self.rows[s]) + len(new):
                    self.table[s].append(self.take())
        except ValueError:
            self.uses, self.table = before
            return False
        for s, new in zip(seqs, tokens):
            self.rows[s] = self.rows[s] + list(new)
        return True

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.table[b], self.rows[b] = list(self.table[a]), list(self.rows[a])
            for p in self.table[b]:
                if p >= 0:
                    self.uses[p] += 1

    def copy(self, src, dst):
        if sum(p >= 0 for a in src for p in self.table[a]) > self.free_pages():
            return False
        for a, b in zip(src, dst):
            self.table[b] = [-1 if p < 0 else self.take() for p in self.table[a]]
            self.rows[b] = list(self.rows[a])
        return True

    def keep(self, seqs, starts, index):
        """index[i]: the positions that sequence seqs[i] keeps behind its first starts[i] tokens."""
        plan, need = [], 0
        for s, start, idx in zip(seqs, starts, index):
            first, end = start // self.T, -(-(start + len(idx)) // self.T)
            fresh = len(idx) > self.IN_PLACE or (len(idx) > 0 and any(self.uses[p] > 1 for p in self.table[s][first:end]))
            plan.append((s, start, idx, first, end, fresh))
            need += end - first if fresh else 0
        if need > self.free_pages():
            return False
        taken = [[self.take() for _ in range(end - first)] if fresh else None for _, _, _, first, end, fresh in plan]
        for (s, start, idx, first, end, fresh), pages in zip(plan, taken):
            old = self.table[s]
            if fresh:
                self.drop(old[first:])
                self.table[s] = old[:first] + pages
            else:
                self.drop(old[end:])
                self.table[s] = old[:end]
            self.rows[s] = self.rows[s][:start] + [self.rows[s][i] if 0 <= i < len(self.rows[s]) else 0 for i in idx]
        return True

    def trim(self, seqs, window, sinks):
        for s in seqs:
            n = len(self.rows[s])
            for p in range(len(self.table[s])):
                if p * self.T >= sinks and (p + 1) * self.T <= n - window + 1 and self.table[s][p] >= 0:
                    self.drop([self.table[s][p]])
                    self.table[s][p] = -1

    def free(self, seqs):
        for s in seqs:
            self.drop(self.table[s])
            self.table[s], self.rows[s] = [], []

    def pack(self):
        used = self.n_pages - self.free_pages()
        holes = [p for p in range(used) if self.uses[p] == 0]
        to = dict(zip([p for p in range(used, self.n_pages) if self.uses[p]], holes))
        for a, b in to.items():
            self.uses[b], self.uses[a] = self.uses[a], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return used
