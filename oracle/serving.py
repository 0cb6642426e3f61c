"""Oracle of the serving calls (include/pkv.h, "Serving from a paged cache"):
rows quantised into a paged cache, read back, and attention over it.

Plain NumPy in fp64, one row and one head at a time.  Test infrastructure only;
imports nothing from the package.  A cache is a dict with the arrays the
library sees:

* tag FP16: ``kv``, the K and the V cache, uint16 bits ``[pool_pages][P][H][D]``;
* other tags: ``codes`` uint8 ``[pool_pages][H][K tile | V tile]`` and
  ``scales`` uint16 bits ``[pool_pages][H][2][P][2]``.
"""
from __future__ import annotations

import numpy as np

from .quantize import KEY_BITS, VALUE_BITS, cache_values, f16_ceil, f16_floor

TAG_FP16 = 0


def quantise_row(x, bits):
    """fp64 values [D] -> (codes [D], scale, zero)."""
    value = lambda b: float(b.astype(np.uint16).view(np.float16)[0])  # noqa: E731
    zero = value(f16_floor(np.array([x.min() + 0.0])))
    scale = value(f16_ceil(np.array([(x.max() - zero + 0.0) / (2 ** bits - 1)])))
    if scale == 0.0:
        return np.zeros(x.size, np.uint8), scale, zero
    return np.clip(np.rint((x - zero) / scale), 0, 2 ** bits - 1).astype(np.uint8), scale, zero


def tile_bounds(tag, page, dim, which):
    """Byte range of the K (0) or V (1) tile of one head of a page."""
    kb, vb = page * dim * KEY_BITS[tag] // 8, page * dim * VALUE_BITS[tag] // 8
    return (0, kb) if which == 0 else (kb, kb + vb)


def places(token_start, kv_lens, page_table, page, pool_pages, positions, num_tokens):
    """For each row: (sequence, position, physical page or -1, slot); sequence -1 for rows of no sequence."""
    out = [(-1, -1, -1, 0)] * num_tokens
    for s in range(len(kv_lens)):
        for i in range(token_start[s], token_start[s + 1]):
            pos = int(positions[i]) if positions is not None else int(kv_lens[s]) - (token_start[s + 1] - i)
            phys = -1
            if pos >= 0 and pos // page < page_table.shape[1]:
                phys = int(page_table[s, pos // page])
                phys = phys if 0 <= phys < pool_pages else -1
            out[i] = (s, pos, phys, pos % page if pos >= 0 else 0)
    return out


def append(cache, tag, page, where, k_bits, v_bits, dtype):
    """Write rows (uint16 bits [tokens][H][D]) at ``where`` (of :func:`places`) into the cache, in place."""
    for which, rows in enumerate((k_bits, v_bits)):
        bits = (KEY_BITS, VALUE_BITS)[which][tag]
        for i, (s, pos, phys, slot) in enumerate(where):
            if s < 0 or phys < 0:
                continue
            for h in range(rows.shape[1]):
                if tag == TAG_FP16:
                    cache["kv"][which][phys, slot, h] = rows[i, h]
                    continue
                codes, scale, zero = quantise_row(cache_values(rows[i, h], dtype), bits)
                lo, hi = tile_bounds(tag, page, codes.size, which)
                tile = cache["codes"][phys, h, lo:hi].reshape(page, -1)
                tile[slot] = codes if bits == 8 else codes[0::2] | (codes[1::2] << 4)
                cache["scales"][phys, h, which, slot] = np.array([scale, zero], np.float16).view(np.uint16)


def row(cache, tag, page, dtype, which, phys, slot, head):
    """One row of the cache as fp64: (values, |value| without its zero around mid-code, that zero)."""
    if tag == TAG_FP16:
        x = cache_values(cache["kv"][which][phys, slot, head], dtype)
        return x, np.abs(x), 0.0
    bits = (KEY_BITS, VALUE_BITS)[which][tag]
    dim = cache["codes"].shape[2] * 8 // (page * (KEY_BITS[tag] + VALUE_BITS[tag]))
    lo, hi = tile_bounds(tag, page, dim, which)
    raw = cache["codes"][phys, head, lo:hi].reshape(page, -1)[slot]
    codes = raw.astype(np.float64) if bits == 8 else np.stack([raw & 15, raw >> 4], 1).reshape(-1).astype(np.float64)
    scale, zero = cache["scales"][phys, head, which, slot].view(np.float16).astype(np.float64)
    mid = 2 ** (bits - 1)
    return codes * scale + zero, np.abs(codes - mid) * scale, abs(zero + mid * scale)


def attend(cache, tag, page, dtype, where, kv_lens, page_table, pool_pages, q_bits, heads, scale, window, sinks):
    """Attention of rows ``q_bits`` (uint16 [tokens][Hq][D]).  Returns fp64 (out, lse) and what error bounds need:
    ``mass`` = sum p |v - zero| / sum p, ``whole`` = sum p (|v - zero| + |zero|) / sum p, both [tokens][Hq][D], and
    ``reach`` [tokens][Hq] = the largest scale * (sum |q k| over channels) of what a row sees."""
    q = cache_values(q_bits, dtype)
    tokens, hq, dim = q.shape
    group = hq // heads
    out, mass, whole = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((tokens, hq), -np.inf), np.zeros((tokens, hq))
    rows = {}
    for i, (s, pos, _, _) in enumerate(where):
        if s < 0:
            continue
        seen = [t for t in range(min(int(kv_lens[s]), pos + 1)) if not window or pos - t < window or t < sinks]
        seen = [(t, int(page_table[s, t // page])) for t in seen if t // page < page_table.shape[1]]
        seen = [(t, p) for t, p in seen if 0 <= p < pool_pages]
        if not seen:
            continue
        for h in range(heads):
            key = (s, h)
            for t, p in seen:
                if (key, t) not in rows:
                    rows[key, t] = (row(cache, tag, page, dtype, 0, p, t % page, h)[0],
                                    row(cache, tag, page, dtype, 1, p, t % page, h))
            k = np.stack([rows[key, t][0] for t, _ in seen])
            v, free, zero = (np.stack([np.asarray(rows[key, t][1][j]) for t, _ in seen]) for j in range(3))
            free, zero = free.reshape(len(seen), dim), zero.reshape(len(seen), 1)
            for g in range(group):
                x = q[i, h * group + g]
                score = scale * (k @ x)
                top = score.max()
                p = np.exp(score - top)
                total = p.sum()
                at = h * group + g
                out[i, at] = p @ v / total
                mass[i, at] = p @ free / total
                whole[i, at] = p @ (free + zero) / total
                lse[i, at] = top + np.log(total)
                reach[i, at] = scale * (np.abs(k) @ np.abs(x)).max()
    return out, lse, mass, whole, reach
