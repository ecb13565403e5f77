"""Measured cases of the state operators: linear attention with a decay for each head, its gradient, its states in a cache, and the
selection of a beam search that reorders them.

A case is a dict of plain values.  ``what`` names the path:

* ``train``: linear attention of whole sequences, forward and backward (``carry``: from a given state, to a final one, both with
  gradients);
* ``attend``: new tokens of some sequences go through a layer whose states a cache holds (``new`` = 1: a decoding step; more: a
  prompt or, where ``held``, a piece of one);
* ``reorder``: in each group of sequences every one goes on from the state of its parent;
* ``select``: the ``k`` best continuations of each group's beams over a vocabulary.

The head dimension is 128, activations are bfloat16, states and decays float32.
"""

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def tokens_case(name, what, seqs, new, q_heads, kv_heads, **more):
    return dict({"name": name, "what": what, "seqs": seqs, "new": new, "q_heads": q_heads, "kv_heads": kv_heads, "ragged": False}, **more)


def listed():
    return [
        # a training batch of short odd sequences, cut out of longer ones: states come in and go out
        tokens_case("train short", "train", 2, 1531, 6, 6, ragged=True, carry=True),
        # long sequences, four query heads to a key head
        tokens_case("train grouped", "train", 1, 16384, 32, 8, carry=False),
        # a training batch with as many key heads as query heads
        tokens_case("train long", "train", 2, 8192, 32, 32, carry=False),
        # a long prompt at once
        tokens_case("prompt long", "attend", 1, 32768, 16, 16, held=False),
        # pieces of prompts of several streams, odd lengths
        tokens_case("prompt pieces", "attend", 5, 700, 12, 12, held=True, ragged=True),
        # one sequence, one token: latency and launches
        tokens_case("step one", "attend", 1, 1, 4, 4, held=True),
        # a serving batch's decoding step
        tokens_case("step batch", "attend", 64, 1, 64, 32, held=True),
        # a serving batch that takes a few drafted tokens each
        tokens_case("step drafts", "attend", 24, 7, 16, 8, held=True, ragged=True),
        # one request's beams change places
        {"name": "reorder one", "what": "reorder", "groups": 1, "beams": 4, "layers": 2, "kv_heads": 4},
        # a serving batch's beams, several layers
        {"name": "reorder batch", "what": "reorder", "groups": 16, "beams": 5, "layers": 4, "kv_heads": 8},
        # one request with few beams, a small vocabulary: latency
        {"name": "select one", "what": "select", "groups": 1, "beams": 4, "vocab": 16001, "k": 4, "type": "fp32"},
        # a serving batch over a large vocabulary
        {"name": "select batch", "what": "select", "groups": 32, "beams": 8, "vocab": 131072, "k": 16, "type": "bf16"},
    ]


MOST = 6.5e8                                               # bytes and flops / 150 of a pass


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        what = rng.choice(["train", "train", "train", "attend", "attend", "attend", "reorder", "select", "select"])
        kv = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 32])
        q = kv * rng.choice([1, 1, 1, 2, 3, 4, 8])
        ragged = rng.random() < 0.5
        if what == "train":
            c = tokens_case("", what, rng.randint(1, 4), log_int(1, 16384), q, kv, ragged=ragged, carry=rng.random() < 0.5)
        elif what == "attend":
            new = rng.choice([1, 1, rng.randint(2, 40), log_int(41, 32768)])
            c = tokens_case("", what, log_int(1, 64), new, q, kv, held=rng.random() < 0.6, ragged=ragged)
        elif what == "reorder":
            c = {"name": "", "what": what, "groups": log_int(1, 32), "beams": rng.randint(2, 32), "layers": rng.randint(1, 4), "kv_heads": kv}
        else:
            c = {"name": "", "what": what, "groups": log_int(1, 64), "beams": rng.randint(1, 32), "vocab": log_int(1000, 200000),
                 "k": rng.choice([1, rng.randint(2, 16), rng.randint(17, 64)]), "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
        del c["name"]
        w = work(c)
        if w["bytes"] + w["flops"] / 150 <= MOST:
            return c


# ---- sizes and inputs -----------------------------------------------------------

def counts(c):
    """(New) tokens of each sequence."""
    n = c["new"]
    return [n - (7919 * i) % (n // 2 + 1) if c["ragged"] else n for i in range(c["seqs"])]


class Draws:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def uniform(self, lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(shape, generator=self.gen, device="cuda")

    def feature(self, *shape):
        """Queries and keys behind an activation: mostly of one sign."""
        return torch.nn.functional.silu(1.5 * self.normal(*shape)).to(torch.bfloat16)

    def value(self, *shape):
        return self.normal(*shape).to(torch.bfloat16)

    def decay(self, heads):
        """Log decays: heads that forget within a token or so, and heads that remember thousands."""
        return -self.uniform(math.log(2e-4), 0.0, heads).exp()


def inputs(c, seed):
    """Everything drawn from the seed, in one order."""
    d, s = Draws(seed), {}
    if c["what"] == "reorder":
        s["state"] = d.normal(c["layers"], c["groups"] * c["beams"], c["kv_heads"], D, D)
        s["parents"] = torch.randint(0, c["beams"], (c["groups"], c["beams"]), generator=d.gen, device="cuda", dtype=torch.int32)
        return s
    if c["what"] == "select":
        G, W = c["groups"], c["beams"]
        s["logits"] = (2.5 * d.normal(G, W, c["vocab"])).to(TYPES[c["type"]])
        s["scores"] = d.uniform(-30.0, -25.0, G, W)
        first = torch.arange(G, device="cuda") % 5 == 4    # requests in their first step: one beam
        s["scores"][first, 1:] = -math.inf
        s["done"] = d.uniform(0.0, 1.0, G, W) < 0.1        # hypotheses that ended
        s["end"] = 2
        return s
    Hq, Hk = c["q_heads"], c["kv_heads"]
    shape = (c["seqs"], c["new"]) if c["what"] == "train" else (sum(counts(c)),)
    s["q"], s["k"], s["v"] = d.feature(*shape, Hq, D), d.feature(*shape, Hk, D), d.value(*shape, Hk, D)
    s["decay"] = d.decay(Hk)
    if c["what"] == "train":
        s["do"] = d.value(*shape, Hq, D)
        s["state"] = d.normal(c["seqs"], Hk, D, D) if c["carry"] else None
        s["dfinal"] = d.normal(c["seqs"], Hk, D, D) if c["carry"] else None
    else:
        s["state"] = d.normal(c["seqs"], Hk, D, D) if c["held"] else torch.zeros((c["seqs"], Hk, D, D), device="cuda")
    s["lengths"] = torch.tensor(counts(c), dtype=torch.int32, device="cuda")
    return s


def prepare(c, seed):
    s = inputs(c, seed)
    s["case"] = c
    if c["what"] in ("train", "select"):
        if not c.get("ragged"):
            s["lengths"] = None
        return s
    layers = c.get("layers", 1)
    n = c["groups"] * c["beams"] if c["what"] == "reorder" else c["seqs"]
    s["ids"] = list(range(n))
    if c["what"] == "attend":
        s["counts"] = counts(c)
    if own:
        import paper_2606_09150_amd as P
        s["cache"] = P.StateCache(layers, c["kv_heads"], n)
        s["cache"].extend(s["ids"], [1] * n)               # sequences that hold something
        s["cache"].states_view().copy_(s["state"])
        s["state"] = None
    return s


# ---- one pass -----------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"train": plain_train, "attend": plain_attend, "reorder": plain_reorder, "select": plain_select}[c["what"]](s)
    import paper_2606_09150_amd as P
    if c["what"] == "select":
        scores, parents, tokens = P.beam_select(s["logits"], s["scores"], c["k"], done=s["done"], end=s["end"])
        return {"scores": scores, "parents": parents, "tokens": tokens}
    if c["what"] == "reorder":
        s["cache"].reorder(s["ids"], s["parents"])
        return {"state": s["cache"].states_view()}
    if c["what"] == "attend":
        if not c["held"]:
            s["cache"].free(s["ids"])                      # an earlier pass's prompts leave
        s["cache"].extend(s["ids"], s["counts"])
        o = s["cache"].attention(0, s["q"], s["k"], s["v"], s["decay"])
        return {"o": o, "state": s["cache"].states_view()[0]}
    q, k, v, do, g = s["q"], s["k"], s["v"], s["do"], s["decay"]
    if not c["carry"]:
        o = P.linear_attention(q, k, v, g, lengths=s["lengths"])
        dq, dk, dv = P.linear_attention_bwd(q, k, v, do, g, lengths=s["lengths"])
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    o, final = P.linear_attention(q, k, v, g, lengths=s["lengths"], state=s["state"], final=True)
    dq, dk, dv, dstate = P.linear_attention_bwd(q, k, v, do, g, lengths=s["lengths"], state=s["state"], dfinal=s["dfinal"])
    return {"o": o, "final": final, "dq": dq, "dk": dk, "dv": dv, "dstate": dstate}


# ---- the plain form: chunks of tokens, products in float32 ---------------------------

CHUNK = 128


def power(g, n):
    """exp(g n), float32, from the product in float64 (which float32 would round before it is exponentiated)."""
    return (g.double() * n).exp().float()


def product(a, b):
    """Batched product of the last two axes, each operand laid out as it is multiplied."""
    return torch.matmul(a.contiguous(), b.contiguous())


class Chunks:
    """Tensors [B, n, heads, D] as chunks [B, Hk, chunks, C * group, D] in float32, with padding as zeros, and the decays between
    their places."""

    def __init__(self, g, n, lengths, kv_heads):
        self.C = min(CHUNK, n)
        self.nc, self.n, self.Hk = -(-n // self.C), n, kv_heads
        self.g = g.view(-1, 1, 1)                          # [Hk, 1, 1]
        self.at = torch.arange(self.nc * self.C, device="cuda").view(self.nc, self.C)
        self.len = None if lengths is None else lengths.long()

    def split(self, x):
        B, G = x.shape[0], x.shape[2] // self.Hk
        x = x.float()
        if self.len is not None:
            x = x * (self.at.view(-1)[:self.n] < self.len[:, None])[:, :, None, None]
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, self.nc * self.C - self.n))
        x = x.view(B, self.nc, self.C, self.Hk, G, D).permute(0, 3, 1, 2, 4, 5)
        return x.reshape(B, self.Hk, self.nc, self.C * G, D)

    def join(self, x):
        """Chunks back as [B, n, heads, D] bfloat16."""
        B, G = x.shape[0], x.shape[3] // self.C
        x = x.view(B, self.Hk, self.nc, self.C, G, D).permute(0, 2, 3, 1, 4, 5)
        return x.reshape(B, self.nc * self.C, self.Hk * G, D)[:, :self.n].to(torch.bfloat16)

    def rows(self, n, group):
        """A weight exp(g n) for each row of a chunk, n [.., C]."""
        return power(self.g, n).repeat_interleave(group, -1).unsqueeze(-1)

    def inside(self, group_rows, group_columns):
        """exp(g (t - j)) of a chunk's places, 0 above the diagonal."""
        i = torch.arange(self.C, device="cuda")
        t, j = i.repeat_interleave(group_rows), i.repeat_interleave(group_columns)
        age = t[:, None] - j[None, :]
        return torch.where(age >= 0, power(self.g, age.clamp(min=0)), 0.0).unsqueeze(1)

    def between(self):
        """[Hk, nc, nc]: exp(g C (c - 1 - i)) for chunks i before c, else 0."""
        c = torch.arange(self.nc, device="cuda")
        gap = c[:, None] - 1 - c[None, :]
        return torch.where(gap >= 0, power(self.g, self.C * gap.clamp(min=0)), 0.0)

    def local(self, a, b, n, group):
        """Per chunk the sum of exp(g n) a b^T, [B, Hk, nc, D, D]."""
        return product((a * self.rows(n, group)).transpose(-1, -2), b)

    def carried(self, local, mix):
        B = local.shape[0]
        return product(mix, local.reshape(B, self.Hk, self.nc, D * D)).view(B, self.Hk, self.nc, D, D)

    def left(self, B):
        """Tokens of a sequence behind each place, [B, 1, nc, C] (negative: padding)."""
        last = torch.full((B,), self.n, device="cuda") if self.len is None else self.len
        return last.view(B, 1, 1, 1) - 1 - self.at


def forward(z, q, k, v, state):
    """(o, chunks' first states) of split tensors."""
    i = torch.arange(z.C, device="cuda")
    G = q.shape[3] // z.C
    starts = z.carried(z.local(k, v, z.C - 1 - i, 1), z.between())
    if state is not None:
        starts = starts + power(z.g, z.at[:, :1]).unsqueeze(-1) * state[:, :, None]
    p = product(q, k.transpose(-1, -2)) * z.inside(G, 1)
    return SCALE * (product(p, v) + product(q * z.rows(i + 1, G), starts)), starts


def final_state(z, k, v, state):
    B = k.shape[0]
    left = z.left(B)
    w = torch.where(left >= 0, power(z.g, left.clamp(min=0)), 0.0).unsqueeze(-1)
    final = product((k * w).flatten(2, 3).transpose(-1, -2), v.flatten(2, 3))
    if state is not None:
        final = final + power(z.g, left[:, :, :1, :1] + 1) * state
    return final


def plain_train(s):
    c = s["case"]
    g, state, dfinal = s["decay"], s["state"], s["dfinal"]
    z = Chunks(g, c["new"], s["lengths"], c["kv_heads"])
    q, k, v, do = (z.split(s[name]) for name in ("q", "k", "v", "do"))
    B, G = c["seqs"], c["q_heads"] // c["kv_heads"]
    i = torch.arange(z.C, device="cuda")
    o, starts = forward(z, q, k, v, state)
    out = {"o": z.join(o)}
    if state is not None:
        out["final"] = final_state(z, k, v, state)
    # the states' gradients behind each chunk, from the chunks after it
    local = z.local(q, do, i + 1, G) * SCALE
    ends = z.carried(local, z.between().transpose(-1, -2))
    m = z.inside(G, 1) * SCALE
    dp = product(do, v.transpose(-1, -2)) * m
    p = product(q, k.transpose(-1, -2)) * m
    dq = product(dp, k) + SCALE * product(do * z.rows(i + 1, G), starts.transpose(-1, -2))
    dk = product(dp.transpose(-1, -2), q) + product(v * z.rows(z.C - 1 - i, 1), ends.transpose(-1, -2))
    dv = product(p.transpose(-1, -2), do) + product(k * z.rows(z.C - 1 - i, 1), ends)
    if dfinal is not None:
        left = z.left(B)
        w = torch.where(left >= 0, power(z.g, left.clamp(min=0)), 0.0).unsqueeze(-1)
        dk = dk + product(v * w, dfinal[:, :, None].transpose(-1, -2))
        dv = dv + product(k * w, dfinal[:, :, None])
        whole = z.rows(z.at + 1, G) * SCALE
        out["dstate"] = product((q * whole).flatten(2, 3).transpose(-1, -2), do.flatten(2, 3)) + power(z.g, left[:, :, :1, :1] + 1) * dfinal
    return dict(out, dq=z.join(dq), dk=z.join(dk), dv=z.join(dv))


def plain_attend(s):
    c = s["case"]
    n, total = c["new"], len(s["q"])
    ends = s["lengths"].cumsum(0)
    i = torch.arange(n, device="cuda")
    rows = ((ends - s["lengths"])[:, None] + i).clamp(max=total - 1)
    z = Chunks(s["decay"], n, s["lengths"], c["kv_heads"])
    q, k, v = (z.split(s[name][rows]) for name in ("q", "k", "v"))
    state = s["state"] if c["held"] else None
    o, _ = forward(z, q, k, v, state)
    s["state"].copy_(final_state(z, k, v, state))
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), s["lengths"], output_size=total)
    at = torch.arange(total, device="cuda") - (ends - s["lengths"])[seq]
    return {"o": z.join(o)[seq, at], "state": s["state"]}


def plain_reorder(s):
    c = s["case"]
    state = s["state"].view(c["layers"], c["groups"], c["beams"], -1)
    at = s["parents"].long() + c["beams"] * torch.arange(c["groups"], device="cuda")[:, None]
    state.copy_(state.flatten(1, 2)[:, at])
    return {"state": s["state"]}


def candidates(s, wide):
    """Every continuation's score [G, W * V]: the sum's logarithm is taken in 64 bits, then each step is rounded to ``wide``."""
    x = s["logits"].to(wide)
    e = s["logits"].double()
    top = e.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    lse = top + (e - top).exp().sum(-1, keepdim=True).log()
    score = s["scores"].to(wide)[..., None]
    got = score + (x - lse.to(wide))
    token = torch.arange(x.shape[-1], device="cuda")
    ended = torch.where(token == s["end"], score, -math.inf)
    got = torch.where(s["done"][..., None], ended, got)
    return got.masked_fill(got.isnan(), -math.inf).flatten(1)


def plain_select(s):
    c = s["case"]
    V, k = c["vocab"], c["k"]
    score = candidates(s, torch.float32)
    bits = score.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)        # ordered as the scores are; the lowest place first among equals
    place = torch.arange(score.shape[1], device="cuda")
    best = (order * (1 << 32) + (0x7FFFFFFF - place)).topk(min(k, score.shape[1]), dim=1).indices
    found = score.gather(1, best)
    there = found > -math.inf
    out = {"scores": found, "parents": torch.where(there, best // V, -1).int(), "tokens": torch.where(there, best % V, -1).int()}
    more = (0, k - best.shape[1])
    return {name: torch.nn.functional.pad(x, more, value=-math.inf if name == "scores" else -1) for name, x in out.items()}


# ---- what a pass cannot do without ------------------------------------------------

def work(c):
    square = 4 * D * D                                     # bytes of a state
    if c["what"] == "select":
        G, W, k = c["groups"], c["beams"], c["k"]
        size = 4 if c["type"] == "fp32" else 2
        return {"bytes": G * (W * c["vocab"] * size + 5 * W + 12 * k), "flops": 5 * G * W * c["vocab"]}
    if c["what"] == "reorder":
        W = c["beams"]
        moved = W - 1                                      # expected of random parents: those that change, and who is read for them
        read = W * (1 - (1 - 1 / W) ** (W - 1))
        return {"bytes": int(c["groups"] * c["layers"] * c["kv_heads"] * square * (moved + read)), "flops": 0}
    n, Hq, Hk = sum(counts(c)), c["q_heads"], c["kv_heads"]
    states = c["seqs"] * Hk * square
    if c["what"] == "train":
        # q, k, v, do in; o, dq, dk, dv out; per token the states' steps, both ways, and what is read off them
        return {"bytes": n * 256 * (4 * Hq + 4 * Hk) + (4 * states if c["carry"] else 0), "flops": 2 * D * D * n * (3 * Hq + 4 * Hk)}
    return {"bytes": n * 256 * (2 * Hq + 2 * Hk) + states * (2 if c["held"] else 1), "flops": 2 * D * D * n * (Hq + Hk)}


# ---- the same in 64 bits, from the definitions ----------------------------------------

def exact_walk(q, k, v, g, state, step=512):
    """One sequence and head in float64, each token's sum over those before it, in bands of queries: (o, final state)."""
    n, age = q.shape[0], torch.arange(q.shape[0], device="cuda", dtype=torch.float64)
    o = torch.empty_like(q)
    for r in range(0, n, step):
        t = age[r:r + step]
        back = t[:, None] - age[None, :r + len(t)]
        w = torch.where(back >= 0, (g * back.clamp(min=0)).exp(), 0.0)
        o[r:r + len(t)] = ((q[r:r + len(t)] @ k[:r + len(t)].T) * w) @ v[:r + len(t)]
    final = (k * (g * (n - 1 - age)).exp()[:, None]).T @ v
    if state is not None:
        o += (q @ state) * (g * (age + 1)).exp()[:, None]
        final = final + (g * n).exp() * state
    return SCALE * o, final


def exact_back(x, y, z, g, last, step=512):
    """out_j = sum over t >= j of exp(g (t - j)) (x_j . y_t) z_t, and exp(g (n - 1 - j)) last^T x_j."""
    n, at = x.shape[0], torch.arange(x.shape[0], device="cuda", dtype=torch.float64)
    out = torch.empty_like(x)
    for r in range(0, n, step):
        j = at[r:r + step]
        ahead = at[None, r:] - j[:, None]
        w = torch.where(ahead >= 0, (g * ahead.clamp(min=0)).exp(), 0.0)
        out[r:r + len(j)] = SCALE * ((x[r:r + len(j)] @ y[r:].T) * w) @ z[r:]
    if last is not None:
        out += (x @ last) * (g * (n - 1 - at)).exp()[:, None]
    return out


def exact(c, seed):
    if c["what"] == "reorder":
        return None                                        # states are moved, no number is computed
    s = inputs(c, seed)
    if c["what"] == "select":
        best = candidates(s, torch.float64).sort(1, descending=True).values[:, :c["k"]]
        best = torch.nn.functional.pad(best, (0, c["k"] - best.shape[1]), value=-math.inf)
        return {"scores": best, "parents": None, "tokens": None}
    G = c["q_heads"] // c["kv_heads"]
    g, lens = s["decay"].double(), counts(c)
    train = c["what"] == "train"
    have = s["state"] is not None and (train or c["held"])
    carry = train and c["carry"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    final = torch.zeros((c["seqs"], c["kv_heads"], D, D), dtype=torch.float64, device="cuda")
    dq, dk, dv, dstate = torch.zeros_like(o), torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda"), None, torch.zeros_like(final)
    dv, at = torch.zeros_like(dk), 0
    for b, n in enumerate(lens):
        rows = (b, slice(0, n)) if train else (slice(at, at + n),)
        at += n
        for h in range(c["q_heads"]):
            e = h // G
            q, k, v = s["q"][rows + (h,)].double(), s["k"][rows + (e,)].double(), s["v"][rows + (e,)].double()
            S = s["state"][b, e].double() if have else None
            o[rows + (h,)], final[b, e] = exact_walk(q, k, v, g[e], S)
            if train:
                do = s["do"][rows + (h,)].double()
                # a key head's part in its final state counts once
                last = s["dfinal"][b, e].double() if carry and h % G == 0 else None
                dq[rows + (h,)] = exact_walk(do, v, k, g[e], None if S is None else S.T)[0]
                dk[rows + (e,)] += exact_back(v, do, q, g[e], None if last is None else last.T)
                dv[rows + (e,)] += exact_back(k, q, do, g[e], last)
                if carry:
                    t = torch.arange(1, n + 1, device="cuda", dtype=torch.float64)
                    dstate[b, e] += SCALE * (q * (g[e] * t).exp()[:, None]).T @ do
                    if last is not None:
                        dstate[b, e] += (g[e] * n).exp() * last
    if not train:
        return {"o": o, "state": final}
    return dict({"o": o, "dq": dq, "dk": dk, "dv": dv}, **({"final": final, "dstate": dstate} if carry else {}))
