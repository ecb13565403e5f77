"""Torch-facing wrappers of the token operators: a paged cache of tokens with the
attention that reads it, and the same attention of whole sequences for training.

Holds the caller-side device buffers and checks shapes, types, devices and streams;
all computation happens in libuf.so's kernels (include/uft.h has the definitions).
"""

import contextlib
import math

import torch

from . import _lib as L
from . import _tokens as T

D = 128


def _check(t, name, shape, dtype=torch.bfloat16, device=None):
    """A device tensor of this type, shape and device."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor (got {type(t).__name__})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not record: detach it, or call under no_grad")


def _dense(t, name, shape, dtype=torch.bfloat16, device=None):
    _check(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _strides(t, name):
    """Strides (batch, token, head) in elements of a tensor [.., tokens, heads, 128]."""
    if t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    # an axis of one element is never stepped along
    s = [0 if n == 1 else st for n, st in zip(t.shape[:-1], t.stride()[:-1])]
    if t.data_ptr() % 16 or any(x % 8 for x in s):
        raise ValueError(f"{name} must be 16-byte aligned, with strides that are multiples of 8 elements")
    return T.uft_stride(s[0] if len(s) == 3 else 0, s[-2], s[-1])


class _On:
    """The stream of a call: the device is current while it is enqueued, and tensors that the call makes belong to it."""

    def __init__(self, device, stream):
        self.device, self.stream, self.stack = device, stream, None

    def __enter__(self):
        if self.stream is None and torch.cuda.current_device() == self.device.index:
            return torch._C._cuda_getCurrentRawStream(self.device.index)
        if self.stream is not None:
            if not isinstance(self.stream, torch.cuda.Stream):
                raise TypeError("stream must be a torch.cuda.Stream")
            if self.stream.device != self.device:
                raise ValueError(f"stream is on {self.stream.device}, the tensors on {self.device}")
        self.stack = contextlib.ExitStack()
        self.stack.enter_context(torch.cuda.device(self.device))
        if self.stream is not None:
            self.stack.enter_context(torch.cuda.stream(self.stream))
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()


def _numbers(x, name):
    if isinstance(x, torch.Tensor):
        raise TypeError(f"{name} are host integers (got a tensor)")
    return [int(i) for i in x]


class TokenCache:
    """At most ``max_seqs`` sequences of up to ``max_tokens`` tokens, in ``n_pages`` pages of ``page_tokens`` (64 or 128)
    tokens that all ``layers`` share one table of.

    One step of a model: ``extend`` the sequences, then per layer ``write`` the new keys and values and ``attention``.
    Every call takes its work on ``stream`` (default: the current one); calls on one cache are to be ordered."""

    def __init__(self, layers, kv_heads, n_pages, max_seqs, max_tokens, page_tokens=64, head_dim=D, flags=0, device=None):
        self.desc = T.uft_desc(layers, kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_tokens, flags)
        self.dry = bool(flags & L.UF_F_DRYRUN)
        self.pool_bytes = T.uft_pool_bytes(self.desc)
        self.pool = self.table = self.device = None
        if not self.dry:
            dev = torch.device("cuda") if device is None else torch.device(device)
            self.pool = torch.empty(self.pool_bytes, dtype=torch.uint8, device=dev)
            self.device = self.pool.device
            self.table = torch.empty(T.uft_table_bytes(self.desc), dtype=torch.uint8, device=self.device)
            self.n_cu = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.handle = T.uft_create(self.desc, self.pool, self.table)

    def close(self):
        if getattr(self, "handle", None) is not None:
            T.uft_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _on(self, stream):
        return contextlib.nullcontext() if self.dry else _On(self.device, stream)

    # -- state ----------------------------------------------------------------
    def info(self):
        return T.uft_get_info(self.handle)

    def tokens(self, seq):
        return T.uft_seq_tokens(self.handle, seq)

    def pages(self, seq):
        """The page of each ``page_tokens`` tokens of a sequence (-1: trimmed)."""
        return T.uft_seq_pages(self.handle, seq)

    def pages_view(self):
        """All pages, [layers, n_pages, (K, V), kv_heads, page_tokens, head_dim] bfloat16."""
        d = self.desc
        return self.pool.view(torch.bfloat16).view(d.layers, d.n_pages, 2, d.kv_heads, d.page_tokens, d.head_dim)

    # -- pages ------------------------------------------------------------------
    def extend(self, seqs, counts, stream=None):
        """Begin a step: sequence seqs[i] grows by counts[i] tokens."""
        seqs, counts = _numbers(seqs, "seqs"), _numbers(counts, "counts")
        with self._on(stream) as s:
            T.uft_extend(self.handle, seqs, counts, s)

    def write(self, layer, k, v, stream=None):
        """The step's keys and values of a layer, [step tokens, kv_heads, 128] (strided views too)."""
        ks = vs = T.uft_stride(0, 0, 0)
        if not self.dry:
            shape = (self.info().step_tokens, self.desc.kv_heads, D)
            _check(k, "k", shape, device=self.device)
            _check(v, "v", shape, device=self.device)
            ks, vs = _strides(k, "k"), _strides(v, "v")
        with self._on(stream) as s:
            T.uft_write(self.handle, layer, k, ks, v, vs, s)

    def fork(self, src, dst, stream=None):
        """Sequences dst[i] continue src[i] and share its pages until one of them grows."""
        src, dst = _numbers(src, "src"), _numbers(dst, "dst")
        with self._on(stream) as s:
            T.uft_fork(self.handle, src, dst, s)

    def copy(self, src, dst, stream=None):
        """Sequences dst[i] continue src[i], in pages of their own."""
        src, dst = _numbers(src, "src"), _numbers(dst, "dst")
        with self._on(stream) as s:
            T.uft_copy(self.handle, src, dst, s)

    def keep(self, seqs, starts, counts, index=None, stream=None):
        """Sequence seqs[i] keeps its first starts[i] tokens, then the tokens at the next counts[i] positions of ``index``
        (int32, on the device), moved up behind them."""
        seqs, starts, counts = _numbers(seqs, "seqs"), _numbers(starts, "starts"), _numbers(counts, "counts")
        if index is not None and not self.dry:
            _dense(index, "index", (sum(counts),), torch.int32, self.device)
        if index is None and any(counts):
            raise ValueError("counts above 0 need an index")
        with self._on(stream) as s:
            T.uft_keep(self.handle, seqs, starts, counts, None if self.dry else index, s)

    def trim(self, seqs, window, sinks=0, stream=None):
        """Give back the pages that no later query of this window and these sinks sees."""
        seqs = _numbers(seqs, "seqs")
        with self._on(stream) as s:
            T.uft_trim(self.handle, seqs, window, sinks, s)

    def free(self, seqs):
        T.uft_free(self.handle, _numbers(seqs, "seqs"))

    def pack(self, stream=None):
        """Move pages so that those in use come first; returns their number."""
        with self._on(stream) as s:
            return T.uft_pack(self.handle, s)

    # -- attention ----------------------------------------------------------------
    def _attn_desc(self, q_heads, window, sinks, scale, stride=None):
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        return T.uft_attn_desc(q_heads, window, sinks, 0 if self.dry else self.n_cu, scale,
                               T.uft_stride(0, 0, 0) if stride is None else stride)

    def work_bytes(self, q_heads, window=0, sinks=0):
        """Scratch that ``attention`` needs for the present step."""
        return T.uft_attn_work_bytes(self.handle, self._attn_desc(q_heads, window, sinks, None))

    def attention(self, layer, q, window=0, sinks=0, scale=None, tree=None, out=None, lse=False, work=None, stream=None):
        """O [step tokens, q_heads, 128] bf16 (and LSE [step tokens, q_heads] fp32 when ``lse``) of the step's tokens.

        ``window`` 0: all earlier tokens; else the last ``window`` and the first ``sinks`` ones.  ``tree``: int64
        [step tokens], the nodes that each new token sees, as bits.  ``work``: scratch (allocated here when None)."""
        if self.dry:
            desc = self._attn_desc(q.shape[1] if hasattr(q, "shape") else q, window, sinks, scale)
            T.uft_attn(self.handle, layer, desc, None, tree, None, None, None)
            return None
        n = self.info().step_tokens
        _check(q, "q", (n, q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0, D), device=self.device)
        Hq = q.shape[1]
        if tree is not None:
            _dense(tree, "tree", (n,), torch.int64, self.device)
        if out is not None:
            _dense(out, "out", (n, Hq, D), device=self.device)
        if isinstance(lse, torch.Tensor):
            _dense(lse, "lse", (n, Hq), torch.float32, self.device)
        desc = self._attn_desc(Hq, window, sinks, scale, _strides(q, "q"))
        need = T.uft_attn_work_bytes(self.handle, desc)
        if work is not None:
            _dense(work, "work", work.shape, torch.uint8, self.device)
            if work.numel() < need:
                raise ValueError(f"work must have {need} bytes or more")
        with self._on(stream) as s:
            if out is None:
                out = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=self.device)
            if lse is True:
                lse = torch.empty((n, Hq), dtype=torch.float32, device=self.device)
            if work is None and need:
                work = torch.empty(need, dtype=torch.uint8, device=self.device)
            lse = lse if isinstance(lse, torch.Tensor) else None
            T.uft_attn(self.handle, layer, desc, q, tree, out, lse, work, None, s)
        return out if lse is None else (out, lse)


def _window_desc(q, k, v, window, sinks, scale, lengths):
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a tensor [batch, tokens, heads, 128]")
    B, n, Hq, _ = q.shape
    Hk = k.shape[2]
    _check(q, "q", (B, n, Hq, D))
    _check(k, "k", (B, n, Hk, D), device=q.device)
    _check(v, "v", (B, n, Hk, D), device=q.device)
    if lengths is not None:
        _dense(lengths, "lengths", (B,), torch.int32, q.device)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    return T.uft_window_desc(B, n, Hq, Hk, D, window, sinks, scale, _strides(q, "q"), _strides(k, "k"), _strides(v, "v"))


def window_attention(q, k, v, window=0, sinks=0, scale=None, lengths=None, out=None, lse=True, stream=None):
    """O [B, n, q_heads, 128] bf16 (and LSE [B, q_heads, n] fp32 when ``lse``) of whole sequences: each token sees itself and
    the tokens before it, with ``window`` > 0 the last ``window`` and the first ``sinks`` ones.

    q [B, n, q_heads, 128], k and v [B, n, kv_heads, 128] bf16, strided views too; ``lengths`` (int32 [B]): tokens from there
    on are padding, whose rows get O = 0 and LSE = -inf."""
    desc = _window_desc(q, k, v, window, sinks, scale, lengths)
    B, n, Hq = q.shape[:3]
    if out is not None:
        _dense(out, "out", q.shape, device=q.device)
    if isinstance(lse, torch.Tensor):
        _dense(lse, "lse", (B, Hq, n), torch.float32, q.device)
    with _On(q.device, stream) as s:
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        if lse is True:
            lse = torch.empty((B, Hq, n), dtype=torch.float32, device=q.device)
        lse = lse if isinstance(lse, torch.Tensor) else None
        T.uft_window_fwd(desc, q, k, v, lengths, out, lse, s)
    return out if lse is None else (out, lse)


def window_attention_bwd(q, k, v, o, lse, do, window=0, sinks=0, scale=None, lengths=None, work=None, stream=None):
    """(dQ, dK, dV) bf16 of ``window_attention`` from its O and LSE; the other arguments as there."""
    desc = _window_desc(q, k, v, window, sinks, scale, lengths)
    B, n, Hq = q.shape[:3]
    _dense(o, "o", q.shape, device=q.device)
    _dense(do, "do", q.shape, device=q.device)
    _dense(lse, "lse", (B, Hq, n), torch.float32, q.device)
    need = T.uft_window_bwd_work_bytes(desc)
    if work is not None:
        _dense(work, "work", work.shape, torch.uint8, q.device)
        if work.numel() < need:
            raise ValueError(f"work must have {need} bytes or more")
    with _On(q.device, stream) as s:
        dq = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        dk = torch.empty(k.shape, dtype=torch.bfloat16, device=q.device)
        dv = torch.empty(k.shape, dtype=torch.bfloat16, device=q.device)
        if work is None:
            work = torch.empty(need, dtype=torch.uint8, device=q.device)
        T.uft_window_bwd(desc, q, k, v, o, lse, do, lengths, dq, dk, dv, work, None, s)
    return dq, dk, dv
