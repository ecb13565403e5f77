"""Measured cases of the token operators: the paged token cache, attention over it, attention for training.

A case is a dict of plain values.  ``what`` names the path:

* ``attend``: new tokens of some sequences enter the cache and attend over it under a sliding window with sinks
  (``new`` = 1: a decoding step; more: a prompt, or a piece of one);
* ``tree``: the same for a tree of drafted tokens a sequence;
* ``train``: the attention of whole sequences, forward and backward;
* ``accept``, ``compact``, ``branch``: the cache's pages (a draft's accepted path stays; chosen tokens stay; sequences fork).

``seqs`` sequences hold ``tokens`` tokens each (``ragged``: different lengths up to that) and get ``new`` more.
The head dimension is 128, types are bfloat16.
"""

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)


def case(name, what, seqs, tokens, new, q_heads, kv_heads, window=0, sinks=0, **more):
    return dict({"name": name, "what": what, "seqs": seqs, "tokens": tokens, "new": new, "q_heads": q_heads,
                 "kv_heads": kv_heads, "window": window, "sinks": sinks, "ragged": False, "page": 64, "layers": 1}, **more)


def listed():
    return [
        # one sequence, one token, a short cache: latency and launches
        case("decode tiny", "attend", 1, 200, 1, 4, 4),
        # a serving batch's decoding step on odd lengths, heads in groups of four, a window with sinks
        case("decode batch", "attend", 48, 12001, 1, 32, 8, 4096, 4, ragged=True),
        # one token over a long cache: all of it is read
        case("decode long", "attend", 1, 131071, 1, 32, 8, page=128),
        # a long prompt at once under a window
        case("prompt window", "attend", 1, 0, 16384, 32, 8, 4096, 4, page=128),
        # pieces of prompts of several streams, odd lengths, a head of keys for each of queries
        case("prompt pieces", "attend", 5, 2900, 700, 12, 12, 1024, 16, ragged=True),
        # a small draft of one stream
        case("tree one", "tree", 1, 2000, 24, 16, 4),
        # full drafts of a serving batch
        case("tree batch", "tree", 16, 8000, 64, 32, 8, 4096, 4, ragged=True),
        # a training batch of short odd sequences
        case("train short", "train", 2, 1531, 0, 6, 6, 200, 3),
        # long sequences with grouped heads
        case("train long", "train", 1, 16384, 0, 32, 8, 2048, 4),
        # a draft's accepted path stays, four layers, a serving batch
        case("accept", "accept", 32, 1000, 48, 8, 8, layers=4, ragged=True),
        # half of the tokens of long sequences stay, in branches of their own
        case("compact", "compact", 4, 30000, 0, 8, 8),
        # eight continuations of each prompt
        case("branch", "branch", 4, 1000, 1, 8, 8, layers=4, ragged=True, branches=8),
    ]


MOST = {"bytes": 8e8, "flops": 1.0e12}


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        what = rng.choice(["attend", "attend", "attend", "tree", "tree", "train", "train", "accept", "compact", "branch"])
        kv = rng.choice([1, 2, 3, 4, 6, 8])
        q = kv * rng.choice([1, 1, 2, 3, 4, 5, 8])
        window = rng.choice([0, 0, log_int(16, 4096)])
        sinks = rng.choice([0, rng.randint(1, 64)]) if window else 0
        more = {"ragged": rng.random() < 0.5, "page": rng.choice([64, 128])}
        if what == "attend":
            new = rng.choice([1, 1, rng.randint(2, 40), log_int(41, 8192)])
            c = case("", what, log_int(1, 64), log_int(64, 131072), new, q, kv, window, sinks, **more)
        elif what == "tree":
            new = rng.randint(2, 64)
            c = case("", what, log_int(1, 32), log_int(64, 32768), new, q, kv, max(window, 64) if window else 0, sinks, **more)
        elif what == "train":
            c = case("", what, rng.randint(1, 4), log_int(64, 16384), 0, q, kv, window, sinks, ragged=more["ragged"])
        elif what == "branch":
            c = case("", what, rng.randint(1, 8), log_int(64, 8192), rng.randint(1, 3), kv, kv, branches=rng.randint(2, 8),
                     layers=rng.randint(1, 4), **more)
        else:
            c = case("", what, log_int(1, 32), log_int(64, 30000), rng.randint(8, 64) if what == "accept" else 0, kv, kv,
                     layers=rng.randint(1, 4), **more)
        del c["name"]
        w = work(c)
        held = sum(lengths(c)) * kv * 512 * c["layers"]
        if w["bytes"] <= MOST["bytes"] and w["flops"] <= MOST["flops"] and held < 2e9:
            return c


# ---- sizes and inputs -----------------------------------------------------------

def lengths(c):
    """Tokens of each sequence before the call."""
    n = c["tokens"]
    return [n - (7919 * i) % (n // 2 + 1) if c["ragged"] else n for i in range(c["seqs"])]


def counts(c):
    """New tokens of each sequence."""
    n = c["new"]
    return [n - (31 * i) % (n // 2 + 1) if c["ragged"] else n for i in range(c["seqs"])]


class Draws:
    """Seeded activations: normal values, keys with an offset per channel that all tokens of a head share."""

    def __init__(self, c, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
        self.q_heads, self.kv_heads = c["q_heads"], c["kv_heads"]
        self.key_offset = 0.5 * torch.randn((self.kv_heads, D), generator=self.gen, device="cuda")

    def normal(self, *shape):
        return torch.randn(shape + (D,), generator=self.gen, device="cuda")

    def kv(self, *n):
        k = (self.normal(*n, self.kv_heads) + self.key_offset).to(torch.bfloat16)
        return k, self.normal(*n, self.kv_heads).to(torch.bfloat16)

    def q(self, *n):
        return (1.25 * self.normal(*n, self.q_heads)).to(torch.bfloat16)


def trees(c, seed):
    """Per sequence the parents of its drafted tokens (-1: the last token of the cache), in order of depth by depth."""
    gen = torch.Generator()
    gen.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    out = []
    for n in counts(c):
        pick = torch.rand(n, generator=gen).tolist()
        out.append([int(pick[t] * (min(t, 12) + 1)) - 1 + max(0, t - 12) for t in range(n)])
    return out


def ancestors(parents):
    """Per node the nodes it descends from and itself, as bits."""
    bits = []
    for t, p in enumerate(parents):
        bits.append((bits[p] if p >= 0 else 0) | (1 << t))
    return bits


def as_int64(bits):
    return [b - (1 << 64) if b >= (1 << 63) else b for b in bits]


def inputs(c, seed):
    """Everything drawn from the seed, in one order."""
    d, s = Draws(c, seed), {}
    if c["what"] == "train":
        B, L = c["seqs"], c["tokens"]
        s["q"], (s["k"], s["v"]), s["do"] = d.q(B, L), d.kv(B, L), d.normal(B, L, c["q_heads"]).to(torch.bfloat16)
        s["lengths"] = torch.tensor(lengths(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
        return s
    s["held"] = [[d.kv(n) for n in lengths(c)] for _ in range(c["layers"])]
    total = sum(counts(c)) * c.get("branches", 1)
    s["new"] = [d.kv(total) for _ in range(c["layers"])] if total else []
    if c["what"] in ("attend", "tree"):
        s["q"] = d.q(total)
    if c["what"] in ("tree", "accept"):
        s["bits"] = [ancestors(p) for p in trees(c, seed)]
    if c["what"] == "tree":
        s["mask"] = torch.tensor(as_int64(sum(s["bits"], [])), dtype=torch.int64, device="cuda")
    if c["what"] == "accept":                              # the path to the deepest node
        paths = []
        for n, bits in zip(lengths(c), s["bits"]):
            best = max(bits, key=lambda b: bin(b).count("1"))
            paths.append([n + t for t in range(len(bits)) if best >> t & 1])
        s["path_counts"] = [len(p) for p in paths]
        s["index"] = torch.tensor(sum(paths, []), dtype=torch.int32, device="cuda")
    if c["what"] == "compact":
        keep = [torch.randperm(n, generator=d.gen, device="cuda")[:(n + 1) // 2].sort().values for n in lengths(c)]
        s["path_counts"] = [len(k) for k in keep]
        s["index"] = torch.cat(keep).to(torch.int32)
    return s


def sequences(c):
    """Sequence numbers in use, besides those that hold the prompts."""
    extra = {"compact": 1, "branch": c.get("branches", 0)}.get(c["what"], 0)
    return c["seqs"] * (1 + extra)


def pages_needed(c):
    T, n = c["page"], 0
    for held, new in zip(lengths(c), counts(c)):
        n += -(-(held + new) // T) + {"compact": -(-((held + 1) // 2) // T), "branch": c.get("branches", 0) * (1 + -(-new // T))
                                      }.get(c["what"], 0)
    return n + 1


def prepare(c, seed):
    s = inputs(c, seed)
    s["case"] = c
    if c["what"] == "train":
        return s
    if own:
        import paper_2606_09150_amd as P
        most = max(a + b for a, b in zip(lengths(c), counts(c)))
        cache = P.TokenCache(c["layers"], c["kv_heads"], pages_needed(c), sequences(c), most, c["page"])
        cache.pool.zero_()
    elif c["what"] in ("attend", "tree"):
        cache = None                                       # the held keys and values as they are, per sequence
    else:
        cache = Pages(c["layers"], c["kv_heads"], pages_needed(c), sequences(c), c["page"])
    if cache is not None:
        cache.extend(list(range(c["seqs"])), lengths(c))
        for layer, held in enumerate(s["held"]):
            if sum(lengths(c)):
                cache.write(layer, torch.cat([k for k, _ in held]), torch.cat([v for _, v in held]))
        del s["held"]
    s["cache"] = cache
    s["lengths"], s["counts"] = lengths(c), counts(c)
    return s


# ---- one pass -----------------------------------------------------------------

def run(s):
    c = s["case"]
    what = c["what"]
    if what == "train":
        if not own:
            return plain_train(s)
        import paper_2606_09150_amd as P
        o, lse = P.window_attention(s["q"], s["k"], s["v"], c["window"], c["sinks"], lengths=s["lengths"])
        dq, dk, dv = P.window_attention_bwd(s["q"], s["k"], s["v"], o, lse, s["do"], c["window"], c["sinks"],
                                            lengths=s["lengths"])
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if what in ("attend", "tree") and not own:
        return plain_attend(s)
    cache, ids = s["cache"], list(range(c["seqs"]))
    if what in ("attend", "tree"):
        cache.keep(ids, s["lengths"], [0] * len(ids))      # an earlier pass's tokens leave
        cache.extend(ids, s["counts"])
        cache.write(0, *s["new"][0])
        return cache.attention(0, s["q"], c["window"], c["sinks"], tree=s.get("mask"))
    if what == "accept":
        cache.keep(ids, s["lengths"], [0] * len(ids))
        cache.extend(ids, s["counts"])
        for layer, (k, v) in enumerate(s["new"]):
            cache.write(layer, k, v)
        cache.keep(ids, s["lengths"], s["path_counts"], s["index"])
    elif what == "compact":
        other = [len(ids) + i for i in ids]
        cache.fork(ids, other)
        cache.keep(other, [0] * len(ids), s["path_counts"], s["index"])
        cache.free(other)
    else:
        n = c["branches"]
        other = [len(ids) + i * n + b for i in ids for b in range(n)]
        cache.fork([i for i in ids for _ in range(n)], other)
        cache.extend(other, [s["counts"][i] for i in ids for _ in range(n)])
        for layer, (k, v) in enumerate(s["new"]):
            cache.write(layer, k, v)
        cache.free(other)
    return cache.pages_view()


# ---- the plain form -------------------------------------------------------------

def visible(pos, keys, window, sinks):
    """bool [queries, keys] from the positions of both."""
    at, j = pos[:, None], keys[None, :]
    see = j <= at
    if window:
        see &= (at - j < window) | (j < sinks)
    return see


def weights(q, k, see):
    """(softmax weights [kv heads, G, queries, keys], q and k as [kv heads, ...] in float32)."""
    n, m, hk = q.shape[0], k.shape[0], k.shape[1]
    q = q.float().view(n, hk, -1, D).permute(1, 2, 0, 3).contiguous()
    k = k.float().permute(1, 0, 2).contiguous()
    s = torch.bmm(q.view(hk, -1, D), k.transpose(1, 2).contiguous()).view(hk, -1, n, m) * SCALE
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(3, keepdim=True)
    e = (s - top.masked_fill(top == -math.inf, 0.0)).exp()
    total = e.sum(3, keepdim=True)
    return e / total.masked_fill(total == 0, 1.0), q, k


def mix(p, v):
    """Weights times values: float32 [queries, heads, D]."""
    hk, g, n, m = p.shape
    v = v.float().permute(1, 0, 2).contiguous()
    return torch.bmm(p.view(hk, g * n, m), v).view(hk, g, n, D).permute(2, 0, 1, 3).reshape(n, hk * g, D)


def key_ranges(first, last, window, sinks):
    """The keys that some query at first .. last may see: [0, a) and [b, last + 1)."""
    low = max(0, first - window + 1) if window else 0
    return (min(sinks, low), low)


def plain_attend(s):
    c = s["case"]
    W, S, at = c["window"], c["sinks"], 0
    out = torch.empty_like(s["q"])
    new_k, new_v = s["new"][0]
    for i, n in enumerate(s["counts"]):
        (k, v), held, rows = s["held"][0][i], s["lengths"][i], slice(at, at + n)
        k, v, q = torch.cat([k, new_k[rows]]), torch.cat([v, new_v[rows]]), s["q"][rows]
        tree = s["mask"][rows] if c["what"] == "tree" else None
        for r in range(0, n, 1024):
            e = min(n, r + 1024)
            first, last = held + r, held + e - 1
            a, b = key_ranges(held if tree is not None else first, last, W, S)
            keys = torch.cat([torch.arange(a, device="cuda"), torch.arange(b, last + 1, device="cuda")])
            if tree is None:
                see = visible(torch.arange(first, last + 1, device="cuda"), keys, W, S)
            else:
                node = (tree[:, None] >> torch.arange(n, device="cuda")) & 1
                see = visible(held + node.sum(1) - 1, keys, W, S)
                see[:, -n:] = node.bool()
            kk, vv = torch.cat([k[:a], k[b:last + 1]]), torch.cat([v[:a], v[b:last + 1]])
            p, _, _ = weights(q[r:e], kk, see)
            out[at + r:at + e] = mix(p, vv).to(torch.bfloat16)
        at += n
    return out


def plain_train(s):
    c = s["case"]
    W, S = c["window"], c["sinks"]
    out, dq = torch.zeros_like(s["q"]), torch.zeros_like(s["q"])
    dk, dv = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    for b, L in enumerate(lengths(c)):
        gk = torch.zeros((c["kv_heads"], L, D), device="cuda")
        gv = torch.zeros_like(gk)
        for r in range(0, L, 1024):
            e = min(L, r + 1024)
            a, lo = key_ranges(r, e - 1, W, S)
            keys = torch.cat([torch.arange(a, device="cuda"), torch.arange(lo, e, device="cuda")])
            see = visible(torch.arange(r, e, device="cuda"), keys, W, S)
            kk, vv = s["k"][b, keys], s["v"][b, keys]
            p, q, k = weights(s["q"][b, r:e], kk, see)
            o = mix(p, vv)
            out[b, r:e] = o.to(torch.bfloat16)
            hk, g, n, m = p.shape
            do = s["do"][b, r:e].float()
            delta = (do * o).sum(2).view(n, hk, g).permute(1, 2, 0)
            do = do.view(n, hk, g, D).permute(1, 2, 0, 3).contiguous().view(hk, g * n, D)
            p = p.view(hk, g * n, m)
            vt = vv.float().permute(1, 2, 0).contiguous()
            ds = p * (torch.bmm(do, vt) - delta.reshape(hk, g * n, 1))
            dq[b, r:e] = (SCALE * torch.bmm(ds, k)).view(hk, g, n, D).permute(2, 0, 1, 3).reshape(n, hk * g, D).to(torch.bfloat16)
            gk[:, keys] += SCALE * torch.bmm(ds.transpose(1, 2).contiguous(), q.view(hk, g * n, D))
            gv[:, keys] += torch.bmm(p.transpose(1, 2).contiguous(), do)
        dk[b, :L] = gk.permute(1, 0, 2).to(torch.bfloat16)
        dv[b, :L] = gv.permute(1, 0, 2).to(torch.bfloat16)
    return {"o": out, "dq": dq, "dk": dk, "dv": dv}


class Pages:
    """A paged cache in plain operations; the lowest free page is taken first."""

    def __init__(self, layers, kv_heads, n_pages, max_seqs, page):
        self.T = page
        self.pool = torch.zeros((layers, n_pages, 2, kv_heads, page, D), dtype=torch.bfloat16, device="cuda")
        self.uses = [0] * n_pages
        self.table = [[] for _ in range(max_seqs)]
        self.length = [0] * max_seqs

    def take(self):
        page = self.uses.index(0)
        self.uses[page] = 1
        return page

    def drop(self, pages):
        for p in pages:
            self.uses[p] -= 1

    def extend(self, seqs, new):
        self.step = []
        for q, n in zip(seqs, new):
            have, T = self.length[q], self.T
            if n and have % T and self.uses[self.table[q][-1]] > 1:
                old, page = self.table[q][-1], self.take()
                self.pool[:, page, :, :, :have % T] = self.pool[:, old, :, :, :have % T]
                self.uses[old] -= 1
                self.table[q][-1] = page
            while len(self.table[q]) * T < have + n:
                self.table[q].append(self.take())
            self.step += [(self.table[q][j // T], j % T) for j in range(have, have + n)]
            self.length[q] = have + n

    def write(self, layer, k, v):
        at = torch.tensor(self.step, device="cuda")
        self.pool[layer, at[:, 0], 0, :, at[:, 1]] = k
        self.pool[layer, at[:, 0], 1, :, at[:, 1]] = v

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.table[b], self.length[b] = list(self.table[a]), self.length[a]
            for p in self.table[a]:
                self.uses[p] += 1

    def keep(self, seqs, starts, new, index=None):
        T, at, left = self.T, 0, []
        for q, start, n in zip(seqs, starts, new):
            first, end = start // T, -(-(start + n) // T)
            table = self.table[q]
            if n:
                rows = torch.cat([torch.arange(first * T, start, device="cuda"), index[at:at + n].long()])
                held = torch.tensor(table, device="cuda")
                data = self.pool[:, held[rows // T], :, :, rows % T].clone()
                if n > 16 or any(self.uses[p] > 1 for p in table[first:end]):
                    fresh = [self.take() for _ in range(first, end)]
                    left += table[first:]
                    table = table[:first] + fresh
                else:
                    left += table[end:]
                    table = table[:end]
                to = torch.tensor(table, device="cuda")
                rows = torch.arange(first * T, start + n, device="cuda")
                self.pool[:, to[rows // T], :, :, rows % T] = data
            else:
                left += table[end:]
                table = table[:end]
            self.table[q], self.length[q], at = table, start + n, at + n
        self.drop(left)

    def free(self, seqs):
        for q in seqs:
            self.drop(self.table[q])
            self.table[q], self.length[q] = [], 0

    def pages_view(self):
        return self.pool


# ---- what a pass cannot do without ------------------------------------------------

def seen(first, n, window, sinks):
    """Pairs of the n queries from position ``first`` on with the keys they see, and the keys that any of them sees."""
    if not window:
        return n * first + n * (n + 1) // 2, first + n
    pairs = 0
    for i in range(first, first + n):
        pairs += min(i + 1, window) + min(sinks, max(0, i + 1 - window))
    low = max(0, first - window + 1)
    return pairs, min(sinks, low) + first + n - low


def work(c):
    row = 512 * c["kv_heads"] * c["layers"]                # K and V of a token
    if c["what"] == "train":
        n = sum(lengths(c))
        pairs = sum(seen(0, L, c["window"], c["sinks"])[0] for L in lengths(c))
        # q, k, v, do in; o, dq, dk, dv out; two products forward, five backward
        return {"bytes": n * (4 * 256 * c["q_heads"] + 2 * row), "flops": 14 * D * pairs * c["q_heads"]}
    if c["what"] in ("attend", "tree"):
        size, flops = 0, 0
        for held, n in zip(lengths(c), counts(c)):
            if c["what"] == "attend":
                pairs, keys = seen(held, n, c["window"], c["sinks"])
            else:                                          # a node sees the window and its ancestors, a few of the nodes
                reach = min(held, c["window"]) + min(c["sinks"], max(0, held - c["window"])) if c["window"] else held
                pairs, keys = n * (reach + n // 8 + 1), reach + n
            size += keys * row + n * row + 2 * 256 * n * c["q_heads"]
            flops += 4 * D * pairs * c["q_heads"]
        return {"bytes": size, "flops": flops}
    if c["what"] == "accept":
        return {"bytes": 2 * row * (sum(counts(c)) + 6 * c["seqs"]), "flops": 0}
    if c["what"] == "compact":
        return {"bytes": 2 * row * sum((n + 1) // 2 for n in lengths(c)), "flops": 0}
    partial = sum(n % c["page"] + m for n, m in zip(lengths(c), counts(c)))
    return {"bytes": 2 * row * c["branches"] * partial, "flops": 0}


# ---- the same in 64 bits, from the definitions ----------------------------------------

def exact_rows(q, k, v, see):
    """One head in float64: (o, p)."""
    s = ((q @ k.T) * SCALE).masked_fill_(~see, -math.inf)
    p = (s - torch.logsumexp(s, 1, keepdim=True)).exp_()
    p = torch.nan_to_num_(p, nan=0.0)                      # a row that sees nothing
    return p @ v, p


def exact(c, seed):
    if c["what"] not in ("attend", "tree", "train"):
        return None                                        # rows are moved, no number is computed
    s = inputs(c, seed)
    W, S, G = c["window"], c["sinks"], c["q_heads"] // c["kv_heads"]
    step = 512
    if c["what"] == "train":
        out, dq = (torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        for b, L in enumerate(lengths(c)):
            j = torch.arange(L, device="cuda")
            for h in range(c["q_heads"]):
                k, v = s["k"][b, :L, h // G].double(), s["v"][b, :L, h // G].double()
                for r in range(0, L, step):
                    rows = j[r:r + step]
                    # the block's own band of keys, and the sinks where they lie before it
                    low = max(0, r - W + 1) if W else 0
                    band = torch.cat([j[:min(S, low)], j[low:r + len(rows)]])
                    age = rows[:, None] - band[None, :]
                    see = (age >= 0) & ((age < W) | (band[None, :] < S)) if W else age >= 0
                    q, g = s["q"][b, rows, h].double(), s["do"][b, rows, h].double()
                    o, p = exact_rows(q, k[band], v[band], see)
                    ds = p * (g @ v[band].T - (g * o).sum(1, keepdim=True)) * SCALE
                    out[b, rows, h], dq[b, rows, h] = o, ds @ k[band]
                    dk[b, band, h // G] += ds.T @ q
                    dv[b, band, h // G] += p.T @ g
        return {"o": out, "dq": dq, "dk": dk, "dv": dv}
    out, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    new_k, new_v = s["new"][0]
    for i, (held, n) in enumerate(zip(lengths(c), counts(c))):
        k = torch.cat([s["held"][0][i][0], new_k[at:at + n]])
        v = torch.cat([s["held"][0][i][1], new_v[at:at + n]])
        j = torch.arange(held + n, device="cuda")
        for r in range(0, n, step):
            rows = torch.arange(r, min(n, r + step), device="cuda")
            pos = held + rows
            if c["what"] == "tree":
                nodes = torch.tensor([[b >> t & 1 for t in range(n)] for b in s["bits"][i]], dtype=torch.bool, device="cuda")
                pos = held + nodes.sum(1) - 1
            low = max(0, int(pos[0]) - W + 1) if W else 0
            band = torch.cat([j[:min(S, low)], j[low:held + r + len(rows)]])
            age = pos[:, None] - band[None, :]
            see = (age >= 0) & ((age < W) | (band[None, :] < S)) if W else age >= 0
            if c["what"] == "tree":
                see = torch.where(band[None, :] < held, see, nodes[:, (band - held).clamp(min=0)])
            for h in range(c["q_heads"]):
                q = s["q"][at + r:at + r + len(rows), h].double()
                out[at + r:at + r + len(rows), h] = exact_rows(q, k[band, h // G].double(), v[band, h // G].double(), see)[0]
        at += n
    return out
