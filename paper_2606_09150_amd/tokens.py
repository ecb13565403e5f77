"""Torch-facing wrappers of the token operators: a paged cache of tokens with the
attention that reads it, and the same attention of whole sequences for training.

Holds the caller-side device buffers and checks shapes, types, devices and streams;
all computation happens in libuf.so's kernels (include/uft.h has the definitions).
"""

import math
import operator

import torch

from . import _lib as L
from . import _tokens as T

D = 128
SCALE = 1.0 / math.sqrt(D)
_NO_STRIDE = T.uft_stride(0, 0, 0)
_forward_ad = torch.autograd.forward_ad                    # (its level is -1 where no tangents are held)


def _check(t, name, shape, dtype=torch.bfloat16, device=None):
    """A device tensor of this type, shape and device, of which no derivative is recorded."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.shape == shape and not t.requires_grad
            and _forward_ad._current_level < 0):
        return                                           # (device: a GPU's)
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor (got {type(t).__name__})")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not record: detach it, or call under no_grad")
    if _forward_ad._current_level >= 0 and _forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has a tangent, which this call does not carry on: hand over its primal")


def _dense(t, name, shape, dtype=torch.bfloat16, device=None):
    _check(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _int(x, name):
    """An integer that a C int32 holds (ctypes would cut a larger one off)."""
    x = operator.index(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must fit in 32 bits (got {x})")
    return x


def _strides(t, name, dense=None):
    """Strides (batch, token, head) in elements of a tensor [.., tokens, heads, 128]; ``dense`` if it is contiguous."""
    if dense is not None and t.is_contiguous() and t.data_ptr() % 16 == 0:
        return dense
    # an axis of one element is never stepped along
    st = [0 if n == 1 else s for n, s in zip(t.shape, t.stride())]
    if st[-1] != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    if t.data_ptr() % 16 or st[-2] % 8 or st[-3] % 8 or st[0] % 8:
        raise ValueError(f"{name} must be 16-byte aligned, with strides that are multiples of 8 elements")
    return T.uft_stride(st[0] if len(st) == 4 else 0, st[-3], st[-2])


_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (a Stream object costs more than a small call)


def _enqueue(device, stream, call, *tensors):
    """``call`` with the stream's handle; the device is current meanwhile, tensors that it makes belong to the stream, and
    ``tensors``, which it works on, are kept from reuse until the stream is past it."""
    if stream is None and _current_device() == device.index:
        return call(_raw_stream(device.index))
    if stream is None:
        with torch.cuda.device(device):
            return call(_raw_stream(device.index))
    if not isinstance(stream, torch.cuda.Stream):
        raise TypeError("stream must be a torch.cuda.Stream")
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    with torch.cuda.device(device), torch.cuda.stream(stream):
        return call(stream.cuda_stream)


class TokenCache:
    """At most ``max_seqs`` sequences of up to ``max_tokens`` tokens, in ``n_pages`` pages of ``page_tokens`` (64 or 128)
    tokens that all ``layers`` share one table of.

    One step of a model: ``extend`` the sequences, then per layer ``write`` the new keys and values and ``attention``.
    Every call takes its work on ``stream`` (default: the current one); calls on one cache are to be ordered."""

    def __init__(self, layers, kv_heads, n_pages, max_seqs, max_tokens, page_tokens=64, head_dim=D, flags=0, device=None):
        sizes = dict(layers=layers, kv_heads=kv_heads, head_dim=head_dim, page_tokens=page_tokens, n_pages=n_pages,
                     max_seqs=max_seqs, max_tokens=max_tokens)
        self.desc = T.uft_desc(flags=flags, **{name: _int(x, name) for name, x in sizes.items()})
        kv_heads = self.desc.kv_heads
        self.dry = bool(flags & L.UF_F_DRYRUN)
        self.pool_bytes = T.uft_pool_bytes(self.desc)
        self.pool = self.table = self.device = None
        self.n_cu = 0
        if not self.dry:
            dev = torch.device("cuda") if device is None else torch.device(device)
            self.pool = torch.empty(self.pool_bytes, dtype=torch.uint8, device=dev)
            self.device = self.pool.device
            self.table = torch.empty(T.uft_table_bytes(self.desc), dtype=torch.uint8, device=self.device)
            self.n_cu = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.handle = T.uft_create(self.desc, self.pool, self.table)
        self._step, self._need = None, {}
        self._dense = T.uft_stride(0, kv_heads * D, D)

    def close(self):
        if getattr(self, "handle", None) is not None:
            T.uft_destroy(self.handle)
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
        return T.uft_get_info(self.handle)

    def tokens(self, seq):
        return T.uft_seq_tokens(self.handle, _int(seq, "seq"))

    def pages(self, seq):
        """The page of each ``page_tokens`` tokens of a sequence (-1: trimmed)."""
        return T.uft_seq_pages(self.handle, _int(seq, "seq"))

    def pages_view(self):
        """All pages, [layers, n_pages, (K, V), kv_heads, page_tokens, head_dim] bfloat16."""
        d = self.desc
        return self.pool.view(torch.bfloat16).view(d.layers, d.n_pages, 2, d.kv_heads, d.page_tokens, d.head_dim)

    def step_tokens(self):
        """New tokens of the step (0: there is none)."""
        if self._step is None:
            self._step = self.info().step_tokens
        return self._step

    # -- pages ------------------------------------------------------------------
    def extend(self, seqs, counts, stream=None):
        """Begin a step: sequence seqs[i] grows by counts[i] tokens."""
        counts = T.ints(counts)
        self._run(stream, lambda s: T.uft_extend(self.handle, seqs, counts, s))
        self._step = sum(counts)
        self._need = {}

    def write(self, layer, k, v, stream=None):
        """The step's keys and values of a layer, [step tokens, kv_heads, 128] (strided views too)."""
        layer = _int(layer, "layer")
        if self.dry:
            return T.uft_write(self.handle, layer, k, _NO_STRIDE, v, _NO_STRIDE)
        shape = (self.step_tokens(), self.desc.kv_heads, D)
        _check(k, "k", shape, device=self.device)
        _check(v, "v", shape, device=self.device)
        ks, vs = _strides(k, "k", self._dense), _strides(v, "v", self._dense)
        self._run(stream, lambda s: T.uft_write(self.handle, layer, k, ks, v, vs, s), k, v)

    def fork(self, src, dst, stream=None):
        """Sequences dst[i] continue src[i] and share its pages until one of them grows."""
        self._run(stream, lambda s: T.uft_fork(self.handle, src, dst, s))

    def copy(self, src, dst, stream=None):
        """Sequences dst[i] continue src[i], in pages of their own."""
        self._run(stream, lambda s: T.uft_copy(self.handle, src, dst, s))

    def keep(self, seqs, starts, counts, index=None, stream=None):
        """Sequence seqs[i] keeps its first starts[i] tokens, then the tokens at the next counts[i] positions of ``index``
        (int32, on the device), moved up behind them."""
        counts = T.ints(counts)
        if index is not None and not self.dry:
            _dense(index, "index", (sum(counts),), torch.int32, self.device)
        if index is None and any(counts):
            raise ValueError("counts above 0 need an index")
        index = None if self.dry else index
        self._run(stream, lambda s: T.uft_keep(self.handle, seqs, starts, counts, index, s), index)
        self._step, self._need = None, {}

    def trim(self, seqs, window, sinks=0, stream=None):
        """Give back the pages that no query of a later step sees under this window and these sinks.  Call it behind the last
        layer of a step: queries of the step itself see nothing in those pages either, and where they hold tokens of the
        step, it ends."""
        window, sinks = _int(window, "window"), _int(sinks, "sinks")
        self._run(stream, lambda s: T.uft_trim(self.handle, seqs, window, sinks, s))
        self._step, self._need = None, {}

    def free(self, seqs):
        T.uft_free(self.handle, seqs)
        self._step, self._need = None, {}

    def pack(self, stream=None):
        """Move pages so that those in use come first; returns their number."""
        return self._run(stream, lambda s: T.uft_pack(self.handle, s))

    # -- attention ----------------------------------------------------------------
    def work_bytes(self, q_heads, window=0, sinks=0):
        """Scratch that ``attention`` needs for the present step."""
        return T.uft_attn_work_bytes(self.handle, T.uft_attn_desc(_int(q_heads, "q_heads"), _int(window, "window"), _int(sinks, "sinks"), self.n_cu, SCALE, _NO_STRIDE))

    def attention(self, layer, q, window=0, sinks=0, scale=None, tree=None, out=None, lse=False, work=None, stream=None):
        """O [step tokens, q_heads, 128] bf16 (and LSE [step tokens, q_heads] fp32 when ``lse``) of the step's tokens.

        ``window`` 0: all earlier tokens; else the last ``window`` and the first ``sinks`` ones.  ``tree``: int64
        [step tokens], the nodes that each new token sees, as bits.  ``work``: scratch (allocated here when None)."""
        layer, window, sinks = _int(layer, "layer"), _int(window, "window"), _int(sinks, "sinks")
        scale = SCALE if scale is None else scale
        if self.dry:                                     # q: the number of its heads
            T.uft_attn(self.handle, layer, T.uft_attn_desc(q, window, sinks, 0, scale, _NO_STRIDE), None, tree, None, None, None)
            return None
        n = self.step_tokens()
        Hq = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        _check(q, "q", (n, Hq, D), device=self.device)
        if tree is not None:
            _dense(tree, "tree", (n,), torch.int64, self.device)
        if out is not None:
            _dense(out, "out", (n, Hq, D), device=self.device)
        if lse is not True and lse is not False and lse is not None:
            _dense(lse, "lse", (n, Hq), torch.float32, self.device)
        desc = T.uft_attn_desc(Hq, window, sinks, self.n_cu, scale, _strides(q, "q"))
        plan = (Hq, window, sinks, self.n_cu)            # the same for every layer of the step
        need = self._need.get(plan)
        if need is None:
            need = self._need[plan] = T.uft_attn_work_bytes(self.handle, desc)
        if work is not None:
            _dense(work, "work", work.shape, torch.uint8, self.device)
            if work.numel() < need:
                raise ValueError(f"work must have {need} bytes or more")

        def call(s):
            o = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=self.device) if out is None else out
            sums = torch.empty((n, Hq), dtype=torch.float32, device=self.device) if lse is True else None if lse is False else lse
            w = torch.empty(need, dtype=torch.uint8, device=self.device) if work is None and need else work
            T.uft_attn(self.handle, layer, desc, q, tree, o, sums, w, need, s)
            return o if sums is None else (o, sums)

        return self._run(stream, call, q, tree, out, work, lse if isinstance(lse, torch.Tensor) else None)


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
    scale = SCALE if scale is None else scale
    return T.uft_window_desc(B, n, Hq, Hk, D, _int(window, "window"), _int(sinks, "sinks"), scale, _strides(q, "q"), _strides(k, "k"), _strides(v, "v"))


def window_attention(q, k, v, window=0, sinks=0, scale=None, lengths=None, out=None, lse=True, stream=None):
    """O [B, n, q_heads, 128] bf16 (and LSE [B, q_heads, n] fp32 when ``lse``) of whole sequences: each token sees itself and
    the tokens before it, with ``window`` > 0 the last ``window`` and the first ``sinks`` ones.

    q [B, n, q_heads, 128], k and v [B, n, kv_heads, 128] bf16, strided views too; ``lengths`` (int32 [B]): tokens from there
    on are padding, whose rows get O = 0 and LSE = -inf."""
    desc = _window_desc(q, k, v, window, sinks, scale, lengths)
    B, n, Hq = q.shape[:3]
    if out is not None:
        _dense(out, "out", q.shape, device=q.device)
    if lse is not True and lse is not False and lse is not None:
        _dense(lse, "lse", (B, Hq, n), torch.float32, q.device)

    def call(s):
        o = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device) if out is None else out
        sums = torch.empty((B, Hq, n), dtype=torch.float32, device=q.device) if lse is True else None if lse is False else lse
        T.uft_window_fwd(desc, q, k, v, lengths, o, sums, s)
        return o if sums is None else (o, sums)

    return _enqueue(q.device, stream, call, q, k, v, lengths, out, lse if isinstance(lse, torch.Tensor) else None)


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

    def call(s):
        dq = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        dk = torch.empty(k.shape, dtype=torch.bfloat16, device=q.device)
        dv = torch.empty(k.shape, dtype=torch.bfloat16, device=q.device)
        w = torch.empty(need, dtype=torch.uint8, device=q.device) if work is None else work
        T.uft_window_bwd(desc, q, k, v, o, lse, do, lengths, dq, dk, dv, w, need, s)
        return dq, dk, dv

    return _enqueue(q.device, stream, call, q, k, v, o, lse, do, lengths, work)
