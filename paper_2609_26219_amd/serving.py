"""Serving from a paged cache: append rows, read them back, attend over them.

Torch tensors in, torch tensors out; every step runs in libpkv
(``include/pkv.h``), on the current stream.  A program keeps one
:class:`PagedCache` per cache and one :class:`Batch` per set of buffers that it
fills anew each step, and calls

* :func:`append`     write new rows (quantised, where the cache holds codes);
* :func:`read`       read rows back;
* :func:`attention`  attention of new or recomputed rows over the cache, with an
  optional sliding window and sinks;
* :func:`rotate`, :func:`append_rotated`  rows turned to their rotary positions,
  the keys on their way into the cache;
* :func:`attention_weights`, :func:`keep`, :func:`evict`  how much attention cached
  tokens receive, which stay under a budget, and the cache without the others.

Nothing here waits for the device or copies from it.  Several host threads may
use one cache, on one stream or on streams of their own.
"""
from __future__ import annotations

import dataclasses
import math
import threading
from typing import Optional

import torch

from . import binding
from .workloads import (KEY_BITS, KV_PAIRED, KV_SEPARATE, OUT_BF16, OUT_FP16, ROPE_HALF, ROPE_INTERLEAVED, TAG_FP16,
                        VALUE_BITS)

_DTYPES = {torch.float16: OUT_FP16, torch.bfloat16: OUT_BF16}


def _check(status: int, where: str) -> None:
    if status != binding.PKV_OK:
        raise binding.PkvError(status, where)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


@dataclasses.dataclass
class _Geometry:
    num_layers: int
    num_kv_heads: int
    head_dim: int
    page_size: int
    pool_pages: int
    out_dtype: int
    kv_layout: int
    rope_theta: float
    rope_style: int
    rotary_dim: int
    inv_freq: tuple
    block_tokens: int = 32  # of checkpoints; the serving calls have no use for it


class PagedCache:
    """A paged cache of all layers.

    ``tag`` FP16: ``k_cache`` and ``v_cache`` of ``dtype`` (or int16, its bits),
    ``[L, pool_pages, P, H, D]`` (or without L for one layer), two tensors or
    the K and V views of one paired cache (``device.alloc_caches``).  Other
    tags: ``codes`` uint8 ``[L, pool_pages, H, bytes]`` and ``scales``
    float16 ``[L, pool_pages, H, 2, P, 2]`` (or without L), allocated here when
    not given (``pool_pages`` and ``device`` then say how many and where).

    The model's RoPE, for the calls that turn rows, as ``workloads.Shape`` has it: ``rope_style`` ROPE_HALF or
    ROPE_INTERLEAVED, ``rotary_dim`` channels (0: all), pair j's frequency ``inv_freq[j]`` (as
    ``workloads.llama3_inv_freq`` gives for long contexts) or ``rope_theta ** (-2 j / rotary_dim)``; turned pairs are
    multiplied by ``rope_amplitude``."""

    def __init__(self, num_kv_heads: int, head_dim: int, page_size: int, dtype, tag: int, codes=None, scales=None,
                 k_cache=None, v_cache=None, num_layers: int = 1, pool_pages: Optional[int] = None, device="cuda",
                 rope_theta: float = 10000.0, rope_style: int = ROPE_HALF, rotary_dim: int = 0, inv_freq=None,
                 rope_amplitude: float = 1.0):
        _need(dtype in _DTYPES, "dtype is float16 or bfloat16")
        _need(0 <= tag < 4, "tag is a TAG_* value")
        _need(rope_style in (ROPE_HALF, ROPE_INTERLEAVED), "rope_style is ROPE_HALF or ROPE_INTERLEAVED")
        rotary = rotary_dim or head_dim
        _need(rotary % 16 == 0 and 16 <= rotary <= head_dim, "rotary_dim is a multiple of 16, at most head_dim")
        _need(math.isfinite(rope_theta) and rope_theta > 0, "rope_theta is above zero")
        if inv_freq is None:  # (here, that calls need not work them out)
            inv_freq = [rope_theta ** (-2.0 * j / rotary) for j in range(rotary // 2)]
        _need(len(inv_freq) == rotary // 2, f"inv_freq has {rotary // 2} values")
        _need(all(math.isfinite(f) for f in inv_freq) and math.isfinite(rope_amplitude), "frequencies are finite")
        layout = KV_SEPARATE
        if tag == TAG_FP16:
            _need(k_cache is not None and v_cache is not None, "16-bit pages need k_cache and v_cache")
            k = k_cache if k_cache.dim() == 5 else k_cache[None]
            v = v_cache if v_cache.dim() == 5 else v_cache[None]
            num_layers, pool_pages = k.shape[0], k.shape[1]
            rows = (page_size, num_kv_heads, head_dim)
            _need(k.shape == v.shape and tuple(k.shape[2:]) == rows, "caches are [L, pool_pages, P, H, D]")
            _need(all(t.dtype in (dtype, torch.int16, torch.uint16) for t in (k, v)),
                  f"caches hold {dtype} or its bits (int16)")
            page = page_size * num_kv_heads * head_dim
            inner = (num_kv_heads * head_dim, head_dim, 1)
            if k.untyped_storage().data_ptr() == v.untyped_storage().data_ptr() and \
                    v.data_ptr() == k.data_ptr() + 2 * page:
                layout = KV_PAIRED
            each = page * (2 if layout == KV_PAIRED else 1)
            for t in (k, v):
                _need(t.stride()[2:] == inner and (pool_pages == 1 or t.stride(1) == each) and
                      (num_layers == 1 or t.stride(0) == pool_pages * each), "caches are whole or paired")
            k_bytes = binding.cache_nbytes(k, v) if layout == KV_PAIRED else 2 * k.numel()
            self.struct = binding.PkvPagedCache(tag, 0, k.data_ptr(), v.data_ptr(), k_bytes, None, 0, None, 0)
        else:
            size = page_size * head_dim * (KEY_BITS[tag] + VALUE_BITS[tag]) // 8
            if codes is None and scales is None:
                _need(pool_pages is not None, "pool_pages of a new cache")
                codes = torch.zeros((num_layers, pool_pages, num_kv_heads, size), dtype=torch.uint8, device=device)
                scales = torch.zeros((num_layers, pool_pages, num_kv_heads, 2, page_size, 2), dtype=torch.float16,
                                     device=device)
            _need(codes is not None and scales is not None, "codes and scales come together")
            c = codes if codes.dim() == 4 else codes[None]
            s = scales if scales.dim() == 6 else scales[None]
            num_layers, pool_pages = c.shape[0], c.shape[1]
            _need(c.dtype == torch.uint8 and s.dtype == torch.float16, "codes are uint8, scales float16")
            _need(tuple(c.shape[2:]) == (num_kv_heads, size), f"codes are [L, pool_pages, H, {size}]")
            _need(tuple(s.shape) == (num_layers, pool_pages, num_kv_heads, 2, page_size, 2),
                  "scales are [L, pool_pages, H, 2, P, 2]")
            _need(c.is_contiguous() and s.is_contiguous(), "codes and scales are contiguous")
            self.struct = binding.PkvPagedCache(tag, 0, None, None, 0, c.data_ptr(), c.numel(), s.data_ptr(),
                                                2 * s.numel())
        self.codes, self.scales, self.k_cache, self.v_cache = codes, scales, k_cache, v_cache
        self.tag, self.dtype, self.head_dim, self.num_kv_heads = tag, dtype, head_dim, num_kv_heads
        self.num_layers, self.pool_pages, self.page_size = num_layers, pool_pages, page_size
        self.device = (k_cache if tag == TAG_FP16 else codes).device
        _need(self.device.type == "cuda", "the cache is device memory")
        self._index = self.device.index
        self.model = binding.make_model(_Geometry(num_layers, num_kv_heads, head_dim, page_size, pool_pages,
                                                  _DTYPES[dtype], layout, rope_theta, rope_style, rotary_dim,
                                                  tuple(inv_freq)))
        self.rope_amplitude = rope_amplitude
        self._layers = [self._of_layer(layer) for layer in range(num_layers)]
        self._workspace = {}
        self._scratch = threading.Lock()  # held from taking scratch memory until the kernels that use it are enqueued

    def _of_layer(self, layer: int) -> binding.PkvPagedCache:
        struct = binding.PkvPagedCache.from_buffer_copy(self.struct)
        struct.layer = layer
        return struct

    def _at(self, layer: int) -> binding.PkvPagedCache:
        """The cache of one layer as the library takes it.  No call writes to it: threads may be in calls of different
        layers at once."""
        return self._layers[layer] if 0 <= layer < self.num_layers else self._of_layer(-1)  # (the library refuses it)

    def workspace(self, nbytes: int, stream: int) -> int:
        """Address of scratch memory for attention calls on one stream (they follow each other), grown as needed.  A
        captured call gets memory of its graph, so that replays share it with nothing else.  The caller holds
        ``_scratch``: the kernels of two calls on one stream must not be enqueued in turn."""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device).data_ptr()
        held = self._workspace.get(stream)
        if held is None or held[0] < nbytes:
            w = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            held = self._workspace[stream] = (nbytes, w.data_ptr(), w)
        return held[1]


class Batch:
    """The rows of a call (``pkv_batch_t``): int32 device tensors ``token_start`` ``[S + 1]``, ``kv_lens`` ``[S]``,
    ``page_table`` ``[S, pages]`` and, for rows that are not the last ones, ``positions`` ``[num_tokens]``.  Their
    contents may change from call to call; ``max_tokens`` and ``max_kv_len`` bound them (0: no bound known)."""

    def __init__(self, token_start, kv_lens, page_table, num_tokens: int, positions=None, max_tokens: int = 0,
                 max_kv_len: int = 0):
        for t in (token_start, kv_lens, page_table, positions):
            _need(t is None or (t.dtype == torch.int32 and t.is_contiguous()), "batch arrays are contiguous int32")
        _need(page_table.dim() == 2 and page_table.shape[0] == kv_lens.numel(), "page_table is [S, pages]")
        _need(token_start.numel() == kv_lens.numel() + 1, "token_start is [S + 1]")
        _need(positions is None or positions.numel() == num_tokens, "positions is [num_tokens]")
        self.keep = (token_start, kv_lens, page_table, positions)
        self.num_tokens = num_tokens
        self.struct = binding.PkvBatch(kv_lens.numel(), num_tokens, max_tokens, page_table.shape[1], max_kv_len,
                                       token_start.data_ptr(), kv_lens.data_ptr(),
                                       None if positions is None else positions.data_ptr(), page_table.data_ptr())


def _rows(cache: PagedCache, batch: Batch, heads: int, *tensors) -> None:
    """Rows of a call: [num_tokens, heads, D] of the cache's dtype, channels together."""
    shape = (batch.num_tokens, heads, cache.head_dim)
    for t in tensors:
        if t.dtype != cache.dtype or t.shape != shape:
            raise ValueError(f"rows are {list(shape)} of {cache.dtype}")
        if t.stride(2) != 1:
            raise ValueError("the channels of a row are consecutive")


def _strides(t) -> tuple:
    """Token and head stride; where a dimension has one element its stride says nothing."""
    (tokens, heads, dim), (token, head, _) = t.shape, t.stride()
    head = head if heads > 1 else dim
    return (token if tokens > 1 else heads * head), head


def _int32(tokens: int) -> int:
    """A number of tokens for the library: past every sequence where it is past 32 bits, below zero where it is."""
    return max(-1, min(tokens, 0x7FFFFFFF))


def _stream(cache: PagedCache) -> int:
    """The current stream of the cache's device (torch.cuda.current_stream(...).cuda_stream without the object: 0.1 us
    against 1.9)."""
    return torch._C._cuda_getCurrentRawStream(cache._index)


def append(cache: PagedCache, batch: Batch, k, v, layer: int = 0) -> None:
    """Write rows ``k``, ``v`` ``[num_tokens, H, D]`` into the cache at the batch's positions.  Each place is to be
    written by one row of the call: several that differ leave pieces of each there."""
    _rows(cache, batch, cache.num_kv_heads, k, v)
    at = _strides(k)
    _need(at == _strides(v), "k and v have the same strides")
    _check(binding.pkv_cache_append_status(cache.model, cache._at(layer), batch.struct, k.data_ptr(), v.data_ptr(), *at,
                                           _stream(cache)), "pkv_cache_append")


def read(cache: PagedCache, batch: Batch, layer: int = 0, out=None):
    """The batch's rows of the cache, ``(k, v)`` of ``[num_tokens, H, D]`` (into ``out`` if given); a row that is not
    there is zero, rows of no sequence are left as they are."""
    if out is None:
        k = torch.empty((batch.num_tokens, cache.num_kv_heads, cache.head_dim), dtype=cache.dtype, device=cache.device)
        v = torch.empty_like(k)
    else:
        k, v = out
    _rows(cache, batch, cache.num_kv_heads, k, v)
    at = _strides(k)
    _need(at == _strides(v), "k and v have the same strides")
    _check(binding.pkv_cache_read_status(cache.model, cache._at(layer), batch.struct, k.data_ptr(), v.data_ptr(), *at,
                                         _stream(cache)), "pkv_cache_read")
    return k, v


def _per_sequence(batch: Batch, t, what: str) -> Optional[int]:
    """Address of an int32 tensor with a number for each sequence, or None."""
    if t is None:
        return None
    _need(t.dtype == torch.int32 and t.is_contiguous() and t.numel() == batch.struct.num_seqs,
          f"{what} is int32, one for each sequence")
    return t.data_ptr()


def _rotation(cache: PagedCache, batch: Batch, x, out, position_offset):
    """The rotation of rows ``x`` into ``out`` (new if None), and ``out``."""
    heads = x.shape[1]
    if out is None:
        _rows(cache, batch, heads, x)
        out = torch.empty((batch.num_tokens, heads, cache.head_dim), dtype=cache.dtype, device=cache.device)
    else:
        _rows(cache, batch, heads, x, out)
    offset = _per_sequence(batch, position_offset, "position_offset")
    return binding.PkvRotation(heads, cache.rope_amplitude, offset, x.data_ptr(), *_strides(x), out.data_ptr(),
                               *_strides(out)), out


def rotate(cache: PagedCache, batch: Batch, x, out=None, position_offset=None):
    """Rows ``x`` ``[num_tokens, heads, D]`` (queries or keys) turned to the batch's positions by the cache's RoPE, into
    ``out`` (which may be ``x``).  ``position_offset``, int32 ``[S]``, is added to the positions of each sequence: after
    an eviction its rows stand further on than their places in the cache.  Rows at negative positions are
    copied, rows of no sequence left as they are."""
    rotation, out = _rotation(cache, batch, x, out, position_offset)
    _check(binding.pkv_rotate_status(cache.model, batch.struct, rotation, _stream(cache)), "pkv_rotate")
    return out


def append_rotated(cache: PagedCache, batch: Batch, q, k, v, layer: int = 0, out=None, position_offset=None):
    """:func:`rotate` of the queries ``q`` ``[num_tokens, Hq, D]`` and :func:`append` of the keys ``k``, turned alike, and the
    values ``v``, in one kernel.  Returns the turned queries (``out``, which may be ``q``); ``k`` and ``v`` are only
    read."""
    rotation, out = _rotation(cache, batch, q, out, position_offset)
    _rows(cache, batch, cache.num_kv_heads, k, v)
    at = _strides(k)
    _need(at == _strides(v), "k and v have the same strides")
    _check(binding.pkv_cache_append_rotated_status(cache.model, cache._at(layer), batch.struct, k.data_ptr(),
                                                   v.data_ptr(), *at, rotation, _stream(cache)),
           "pkv_cache_append_rotated")
    return out


def attention(cache: PagedCache, batch: Batch, q, scale: Optional[float] = None, window: int = 0, sinks: int = 0,
              layer: int = 0, out=None, return_lse: bool = False):
    """Attention of rows ``q`` ``[num_tokens, Hq, D]`` over the cache, causal by position: a row at position p sees
    tokens t <= p and, with a window, those with p - t < window or t < sinks.  ``scale`` defaults to D ** -0.5.
    Returns ``out`` ``[num_tokens, Hq, D]``, with ``return_lse`` also the rows' log-sum-exp, float32
    ``[num_tokens, Hq]``.  A row that sees nothing gives 0 and -inf.

    How a call is cut follows from its longest sequence of rows: a prompt's chunk and the decode rows of other
    sequences are faster as two calls."""
    heads = q.shape[1]
    if out is None:
        out = torch.empty_like(q)
        _rows(cache, batch, heads, q)
    else:
        _rows(cache, batch, heads, q, out)
    lse = q.new_empty((batch.num_tokens, heads), dtype=torch.float32) if return_lse else None
    a = binding.PkvAttention(heads, _int32(window), _int32(sinks), cache.head_dim ** -0.5 if scale is None else scale,
                             q.data_ptr(), *_strides(q), out.data_ptr(), *_strides(out),
                             lse.data_ptr() if return_lse else None, None, 0)
    stream = _stream(cache)
    struct = cache._at(layer)
    nbytes = binding.pkv_attention_workspace(cache.model, struct, batch.struct, a)
    if nbytes:
        with cache._scratch:
            a.workspace, a.workspace_bytes = cache.workspace(nbytes, stream), nbytes
            status = binding.pkv_attention_status(cache.model, struct, batch.struct, a, stream)
    else:
        status = binding.pkv_attention_status(cache.model, struct, batch.struct, a, stream)
    _check(status, "pkv_attention")
    return (out, lse) if return_lse else out


def _weights(cache: PagedCache, batch: Batch, out, weights=None, decay: float = 0.0) -> binding.PkvWeights:
    """Numbers of cached tokens as the library takes them: float32 ``[S, 1 or H, tokens]``, tokens together."""
    for t in (out, weights):
        if t is not None and (t.dtype != torch.float32 or t.dim() != 3 or t.shape[0] != batch.struct.num_seqs or
                              t.shape[1] not in (1, cache.num_kv_heads) or (t.shape[2] > 1 and t.stride(2) != 1)):
            raise ValueError("weights are float32 [S, 1 or H, tokens], a row's tokens consecutive")
    seqs, heads, tokens = out.shape
    head = out.stride(1) if heads > 1 else tokens
    seq = out.stride(0) if seqs > 1 else heads * head
    _need(weights is None or weights.shape == out.shape, "weights before and after have the same shape")
    if weights is not None:
        _need((heads == 1 or weights.stride(1) == head) and (seqs == 1 or weights.stride(0) == seq),
              "weights before and after have the same strides")
    return binding.PkvWeights(heads, decay, tokens, head, seq, None if weights is None else weights.data_ptr(),
                              out.data_ptr())


def attention_weights(cache: PagedCache, batch: Batch, q, lse, out, weights=None, decay: float = 1.0,
                      scale: Optional[float] = None, window: int = 0, sinks: int = 0, layer: int = 0):
    """The attention weight that each cached token receives from the rows of an :func:`attention` call (the same ``q``,
    ``scale`` and masks, and the ``lse`` that it returned), added to ``decay`` times what it had before:
    ``out = decay * weights + sum``, float32 ``[S, H, tokens]`` for each KV head or ``[S, 1, tokens]`` for all together,
    with as many tokens as the batch's bound.  ``weights`` may be ``out`` (added in place) or None (nothing before).  Tokens
    past ``kv_lens`` are left as they are.  ``scale`` is 2^-64 or more.  Returns ``out``."""
    heads = q.shape[1]
    _rows(cache, batch, heads, q)
    _need(lse.dtype == torch.float32 and lse.shape == (batch.num_tokens, heads) and lse.is_contiguous(),
          "lse is contiguous float32 [num_tokens, Hq]")
    w = _weights(cache, batch, out, weights, decay if weights is not None else 0.0)
    a = binding.PkvAttention(heads, _int32(window), _int32(sinks), cache.head_dim ** -0.5 if scale is None else scale,
                             q.data_ptr(), *_strides(q), None, 0, 0, lse.data_ptr(), None, 0)
    stream = _stream(cache)
    struct = cache._at(layer)
    nbytes = binding.pkv_attention_weights_workspace(cache.model, struct, batch.struct, a, w)
    if nbytes:
        with cache._scratch:
            a.workspace, a.workspace_bytes = cache.workspace(nbytes, stream), nbytes
            status = binding.pkv_attention_weights_status(cache.model, struct, batch.struct, a, w, stream)
    else:
        status = binding.pkv_attention_weights_status(cache.model, struct, batch.struct, a, w, stream)
    _check(status, "pkv_attention_weights")
    return out


def keep(cache: PagedCache, batch: Batch, weights, budget: int, sinks: int = 0, recent: int = 0, budgets=None, out=None):
    """The tokens of each sequence that stay under a ``budget``: the first ``sinks``, the last ``recent``, and of those
    between the ones of the largest ``weights`` (float32 ``[S, 1, tokens]``: one choice for all heads, or
    ``[S, H, tokens]``: each head its own), equal ones lowest index first.  ``budgets``, int32 ``[S]``, sets a sequence's
    own, up to ``budget``.  Returns ``(kept, kept_lens)``, int32 ``[S, 1 or H, budget]``, ascending and then -1, and
    ``[S]`` (``out`` if given, which is neither the batch's lengths nor ``budgets``)."""
    w = _weights(cache, batch, weights, weights)
    if out is None:
        out = (torch.empty((batch.struct.num_seqs, w.heads, max(0, budget)), dtype=torch.int32, device=cache.device),
               torch.empty(batch.struct.num_seqs, dtype=torch.int32, device=cache.device))
    kept = _kept(batch, *out, budgets, _int32(sinks), _int32(recent))
    _need(kept.heads == w.heads and kept.budget == budget, "kept is [S, heads of weights, budget]")
    stream = _stream(cache)
    nbytes = binding.pkv_cache_keep_workspace(cache.model, batch.struct, w, kept)
    if nbytes:
        with cache._scratch:
            kept.workspace, kept.workspace_bytes = cache.workspace(nbytes, stream), nbytes
            status = binding.pkv_cache_keep_status(cache.model, batch.struct, w, kept, stream)
    else:
        status = binding.pkv_cache_keep_status(cache.model, batch.struct, w, kept, stream)
    _check(status, "pkv_cache_keep")
    return out


def _kept(batch: Batch, kept, kept_lens, budgets=None, sinks: int = 0, recent: int = 0) -> binding.PkvKept:
    _need(kept.dtype == torch.int32 and kept.dim() == 3 and kept.shape[0] == batch.struct.num_seqs and
          kept.is_contiguous(), "kept is contiguous int32 [S, 1 or H, budget]")
    return binding.PkvKept(kept.shape[1], kept.shape[2], sinks, recent, _per_sequence(batch, budgets, "budgets"),
                           kept.data_ptr(), _per_sequence(batch, kept_lens, "kept_lens"))


def evict(cache: PagedCache, batch: Batch, kept, kept_lens, weights=None, page_table=None, layer: int = 0) -> None:
    """Move the rows that stay to the front of their sequence: row j becomes row ``kept[s, h, j]``, in place, or with a
    ``page_table`` ``[S, pages]`` of other pages (where the batch's are shared, they keep theirs).  ``weights`` are moved
    alike, in place, and 0 behind the rows that stayed.  The batch's ``kv_lens`` are only read: after the last layer the
    lengths are ``kept_lens``, and what a sequence lost is added to its ``position_offset``."""
    k = _kept(batch, kept, kept_lens)
    w = None if weights is None else _weights(cache, batch, weights)
    _need(page_table is None or (page_table.dtype == torch.int32 and page_table.dim() == 2 and
                                 page_table.is_contiguous() and page_table.shape[0] == batch.struct.num_seqs),
          "page_table is contiguous int32 [S, pages]")
    table, pages = (None, 0) if page_table is None else (page_table.data_ptr(), page_table.shape[1])
    _check(binding.pkv_cache_evict_status(cache.model, cache._at(layer), batch.struct, k, w, table, pages,
                                          _stream(cache)), "pkv_cache_evict")
