"""Serving from a paged cache: append rows, read them back, attend over them.

Torch tensors in, torch tensors out; every step runs in libpkv
(``include/pkv.h``), on the current stream.  A program keeps one
:class:`PagedCache` per cache and one :class:`Batch` per set of buffers that it
fills anew each step, and calls

* :func:`append`     write new rows (quantised, where the cache holds codes);
* :func:`read`       read rows back;
* :func:`attention`  attention of new or recomputed rows over the cache, with an
  optional sliding window and sinks.

Nothing here waits for the device or copies from it.  Several host threads may
use one cache, on one stream or on streams of their own.
"""
from __future__ import annotations

import dataclasses
import threading
from typing import Optional

import torch

from . import binding
from .workloads import KEY_BITS, KV_PAIRED, KV_SEPARATE, OUT_BF16, OUT_FP16, TAG_FP16, VALUE_BITS

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
    block_tokens: int = 32  # of checkpoints; the serving calls have no use for it
    rope_theta: float = 10000.0


class PagedCache:
    """A paged cache of all layers.

    ``tag`` FP16: ``k_cache`` and ``v_cache`` of ``dtype`` (or int16, its bits),
    ``[L, pool_pages, P, H, D]`` (or without L for one layer), two tensors or
    the K and V views of one paired cache (``device.alloc_caches``).  Other
    tags: ``codes`` uint8 ``[L, pool_pages, H, bytes]`` and ``scales``
    float16 ``[L, pool_pages, H, 2, P, 2]`` (or without L), allocated here when
    not given (``pool_pages`` and ``device`` then say how many and where)."""

    def __init__(self, num_kv_heads: int, head_dim: int, page_size: int, dtype, tag: int, codes=None, scales=None,
                 k_cache=None, v_cache=None, num_layers: int = 1, pool_pages: Optional[int] = None, device="cuda"):
        _need(dtype in _DTYPES, "dtype is float16 or bfloat16")
        _need(0 <= tag < 4, "tag is a TAG_* value")
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
                                                  _DTYPES[dtype], layout))
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
