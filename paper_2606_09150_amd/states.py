"""Torch-facing wrappers of the state operators: linear attention with a decay for each head (whole sequences with their
gradient, and over states that a cache holds), and the selection of a beam search.

Holds the caller-side device buffers and checks shapes, types, devices and streams;
all computation happens in libuf.so's kernels (include/ufs.h has the definitions).
"""

import torch

from . import _lib as L
from . import _states as S
from .tokens import D, SCALE, _check, _dense, _enqueue, _int, _strides

_TYPES = {torch.bfloat16: S.UFS_BF16, torch.float16: S.UFS_FP16, torch.float32: S.UFS_FP32}


def _work(work, need, device):
    if work is not None:
        _dense(work, "work", work.shape if isinstance(work, torch.Tensor) else None, torch.uint8, device)
        if work.numel() < need:
            raise ValueError(f"work must have {need} bytes or more")


def _scratch(work, need, like):
    return like.new_empty(need, dtype=torch.uint8) if work is None and need else work


def _states(t, name, shape, device):
    """States [.., kv_heads, 128, 128] float32, contiguous."""
    _dense(t, name, shape, torch.float32, device)
    if t.data_ptr() % 16:
        raise ValueError(f"{name} must be 16-byte aligned")


def _like(t):
    """An uninitialised contiguous tensor of the same shape (half of torch.empty's time from its parts)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _whole_strides(t, name):
    if t.is_contiguous() and not t.data_ptr() % 16:
        _, n, heads, _ = t.shape
        return S.uft_stride(n * heads * D, heads * D, D)
    return _strides(t, name)


def _linear_desc(q, k, v, decay, scale, lengths):
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a tensor [batch, tokens, heads, 128]")
    B, n, Hq, _ = q.shape
    Hk = k.shape[2]
    _check(q, "q", (B, n, Hq, D))
    _check(k, "k", (B, n, Hk, D), device=q.device)
    _check(v, "v", (B, n, Hk, D), device=q.device)
    _dense(decay, "decay", (Hk,), torch.float32, q.device)
    if lengths is not None:
        _dense(lengths, "lengths", (B,), torch.int32, q.device)
    scale = SCALE if scale is None else scale
    return S.ufs_linear_desc(B, n, Hq, Hk, D, scale, _whole_strides(q, "q"), _whole_strides(k, "k"), _whole_strides(v, "v"))


def linear_attention(q, k, v, decay, scale=None, lengths=None, state=None, final=False, out=None, work=None, stream=None):
    """O [B, n, q_heads, 128] bf16 of whole sequences: o_t = scale S_t^T q_t with S_t = exp(decay) S_{t-1} + k_t v_t^T.

    q [B, n, q_heads, 128], k and v [B, n, kv_heads, 128] bf16, strided views too; ``decay`` (fp32 [kv_heads]): log decays, at
    most 0; ``lengths`` (int32 [B]): tokens from there on are padding, whose rows get 0.  ``state`` (fp32 [B, kv_heads, 128 (of
    k), 128 (of v)]): the states before the first token.  ``final``: those behind the last one are wanted too (True, or a
    tensor for them, which may be ``state``); then (O, final) is returned."""
    desc = _linear_desc(q, k, v, decay, scale, lengths)
    B, Hk = q.shape[0], k.shape[2]
    shape = (B, Hk, D, D)
    if state is not None:
        _states(state, "state", shape, q.device)
    if out is not None:
        _dense(out, "out", q.shape, device=q.device)
    if isinstance(final, torch.Tensor):
        _states(final, "final", shape, q.device)
    need = S.ufs_linear_work_bytes(desc)
    _work(work, need, q.device)

    def call(s):
        o = _like(q) if out is None else out
        last = final if isinstance(final, torch.Tensor) else torch.empty(shape, dtype=torch.float32, device=q.device) if final else None
        S.ufs_linear_fwd(desc, q, k, v, decay, lengths, state, o, last, _scratch(work, need, q), need, s)
        return o if last is None else (o, last)

    return _enqueue(q.device, stream, call, q, k, v, decay, lengths, state, out, work, final if isinstance(final, torch.Tensor) else None)


def linear_attention_bwd(q, k, v, do, decay, scale=None, lengths=None, state=None, dfinal=None, work=None, stream=None):
    """(dQ, dK, dV) bf16 of ``linear_attention``, the other arguments as there; (dQ, dK, dV, dState) where it began from a
    ``state``.  ``dfinal`` (fp32, as the states): the gradient of the final states, None where they have none.  Decays are
    constants."""
    desc = _linear_desc(q, k, v, decay, scale, lengths)
    shape = (q.shape[0], k.shape[2], D, D)
    _dense(do, "do", q.shape, device=q.device)
    if state is not None:
        _states(state, "state", shape, q.device)
    if dfinal is not None:
        _states(dfinal, "dfinal", shape, q.device)
    need = S.ufs_linear_bwd_work_bytes(desc)
    _work(work, need, q.device)

    def call(s):
        dq, dk, dv = _like(q), _like(k), _like(v)
        dstate = None if state is None else _like(state)
        S.ufs_linear_bwd(desc, q, k, v, do, decay, lengths, state, dfinal, dq, dk, dv, dstate, _scratch(work, need, q), need, s)
        return (dq, dk, dv) if dstate is None else (dq, dk, dv, dstate)

    return _enqueue(q.device, stream, call, q, k, v, do, decay, lengths, state, dfinal, work)


class StateCache:
    """States of linear attention of at most ``max_seqs`` sequences in ``layers`` layers, [128, 128] float32 a key head.

    One step of a model: ``extend`` the sequences, then ``attention`` once per layer, which moves the layer's states past the
    new tokens.  Every call takes its work on ``stream`` (default: the current one); calls on one cache are to be ordered."""

    def __init__(self, layers, kv_heads, max_seqs, head_dim=D, flags=0, device=None):
        sizes = dict(layers=layers, kv_heads=kv_heads, head_dim=head_dim, max_seqs=max_seqs)
        self.desc = S.ufs_desc(flags=flags, **{name: _int(x, name) for name, x in sizes.items()})
        self.dry = bool(flags & L.UF_F_DRYRUN)
        self.pool_bytes = S.ufs_pool_bytes(self.desc)
        self.pool = self.table = self.device = None
        if not self.dry:
            dev = torch.device("cuda") if device is None else torch.device(device)
            self.pool = torch.empty(self.pool_bytes, dtype=torch.uint8, device=dev)
            self.device = self.pool.device
            self.table = torch.empty(S.ufs_table_bytes(self.desc), dtype=torch.uint8, device=self.device)
        self.handle = S.ufs_create(self.desc, self.pool, self.table)
        self._step = self._need = None
        self._dense = {}

    def _of(self, heads):
        """The strides of contiguous [tokens, heads, 128]."""
        got = self._dense.get(heads)
        if got is None:
            got = self._dense[heads] = S.uft_stride(0, heads * D, D)
        return got

    def close(self):
        if getattr(self, "handle", None) is not None:
            S.ufs_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _run(self, stream, call, *tensors):
        return call(None) if self.dry else _enqueue(self.device, stream, call, self.pool, self.table, *tensors)

    # -- state ----------------------------------------------------------------
    def info(self):
        return S.ufs_get_info(self.handle)

    def tokens(self, seq):
        """Tokens that a sequence has taken (0: its state is zero, whatever lies in its place)."""
        return S.ufs_seq_tokens(self.handle, _int(seq, "seq"))

    def states_view(self):
        """All states, [layers, max_seqs, kv_heads, 128 (of k), 128 (of v)] float32."""
        d = self.desc
        return self.pool.view(torch.float32).view(d.layers, d.max_seqs, d.kv_heads, D, D)

    def step_tokens(self):
        """New tokens of the step (0: there is none)."""
        if self._step is None:
            self._step = self.info().step_tokens
        return self._step

    # -- sequences --------------------------------------------------------------
    def extend(self, seqs, counts, stream=None):
        """Begin a step: sequence seqs[i] grows by counts[i] tokens."""
        counts = S.ints(counts)
        self._step = self._need = None                   # (a failed launch can end the step before)
        self._run(stream, lambda s: S.ufs_extend(self.handle, seqs, counts, s))
        self._step = sum(counts)

    def fork(self, src, dst, stream=None):
        """Sequences dst[i], empty before, continue src[i]: their states are copied."""
        self._run(stream, lambda s: S.ufs_fork(self.handle, src, dst, s))
        self._step = self._need = None

    def reorder(self, seqs, parents, stream=None):
        """Sequence seqs[g * beams + i] goes on from the state of seqs[g * beams + parents[g, i]], in each group g, all
        layers.  ``parents``: int32 [groups, beams] on the device, as ``beam_select`` gives them (a dry run: a shape); one that
        is none of 0 .. beams-1 leaves its sequence as it is."""
        shape = parents if self.dry else parents.shape if isinstance(parents, torch.Tensor) else ()
        if len(shape) != 2:
            raise ValueError("parents must be a tensor [groups, beams]")
        if not self.dry:
            _dense(parents, "parents", shape, torch.int32, self.device)
        seqs = S.ints(seqs)
        if len(seqs) != shape[0] * shape[1]:
            raise ValueError(f"parents of {tuple(shape)} need as many sequences (got {len(seqs)})")
        tensor = None if self.dry else parents
        self._step = self._need = None
        self._run(stream, lambda s: S.ufs_reorder(self.handle, _int(shape[1], "beams"), seqs, tensor, s), tensor)

    def free(self, seqs):
        S.ufs_free(self.handle, seqs)
        self._step = self._need = None

    # -- attention ----------------------------------------------------------------
    def work_bytes(self):
        """Scratch that ``attention`` needs for the present step."""
        if self._need is None:
            self._need = S.ufs_attn_work_bytes(self.handle)
        return self._need

    def attention(self, layer, q, k, v, decay, scale=None, out=None, work=None, stream=None):
        """O [step tokens, q_heads, 128] bf16 of the step's tokens; the layer's states move past them.

        q [step tokens, q_heads, 128], k and v [step tokens, kv_heads, 128] bf16, strided views too; ``decay`` (fp32
        [kv_heads]): log decays, at most 0.  ``work``: scratch (allocated here when None)."""
        layer = _int(layer, "layer")
        scale = SCALE if scale is None else scale
        if self.dry:                                     # q: the number of its heads
            none = S.uft_stride(0, 0, 0)
            S.ufs_attn(self.handle, layer, S.ufs_attn_desc(q, scale, none, none, none), None, k, v, decay, None, None)
            return None
        n, Hk = self.step_tokens(), self.desc.kv_heads
        Hq = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        _check(q, "q", (n, Hq, D), device=self.device)
        _check(k, "k", (n, Hk, D), device=self.device)
        _check(v, "v", (n, Hk, D), device=self.device)
        _dense(decay, "decay", (Hk,), torch.float32, self.device)
        if out is not None:
            _dense(out, "out", (n, Hq, D), device=self.device)
        desc = S.ufs_attn_desc(Hq, scale, _strides(q, "q", self._of(Hq)), _strides(k, "k", self._of(Hk)), _strides(v, "v", self._of(Hk)))
        need = self._need if self._need is not None else self.work_bytes()
        if work is not None:
            _work(work, need, self.device)

        def call(s):
            o = _like(q) if out is None else out
            S.ufs_attn(self.handle, layer, desc, q, k, v, decay, o, _scratch(work, need, q), need, s)
            return o

        return self._run(stream, call, q, k, v, decay, out, work)


def beam_select(logits, scores, k, done=None, end=None, work=None, stream=None):
    """(scores fp32, parents int32, tokens int32), each [groups, k]: of each group's continuations the k of the highest
    scores[w] + log_softmax(logits[w])[t], best first, equal ones by the lowest (w, t).

    logits [groups, beams, vocab] bf16, fp16 or fp32, contiguous along the vocabulary; scores fp32 [groups, beams], -inf for
    a hypothesis that is not in use.  ``done`` (bool or uint8 [groups, beams]): finished hypotheses, which have the one
    continuation ``end``, at the score they have.  Places that no continuation fills get -inf, -1 and -1."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 3:
        raise ValueError("logits must be a tensor [groups, beams, vocab]")
    if logits.dtype not in _TYPES:
        raise TypeError(f"logits must be bfloat16, float16 or float32 (got {logits.dtype})")
    G, W, V = logits.shape
    k, dev = _int(k, "k"), logits.device
    _check(logits, "logits", (G, W, V), logits.dtype)
    if V > 1 and logits.stride(2) != 1:
        raise ValueError("logits must be contiguous along the vocabulary")
    _dense(scores, "scores", (G, W), torch.float32, dev)
    if done is not None:
        _dense(done, "done", (G, W), torch.uint8 if getattr(done, "dtype", None) is torch.uint8 else torch.bool, dev)
        if end is None:
            raise ValueError("done needs end, the token that finished hypotheses go on with")
    strides = [0 if n == 1 else s for n, s in zip(logits.shape, logits.stride())]
    desc = S.ufs_select_desc(G, W, V, k, _TYPES[logits.dtype], 0 if end is None else _int(end, "end"), strides[0], strides[1])
    need = S.ufs_select_work_bytes(desc)
    _work(work, need, dev)

    def call(s):
        best = scores.new_empty((G, k))
        parents, tokens = scores.new_empty((2, G, k), dtype=torch.int32).unbind()
        S.ufs_select(desc, logits, scores, done, best, parents, tokens, _scratch(work, need, logits), need, s)
        return best, parents, tokens

    return _enqueue(dev, stream, call, logits, scores, done, work)
