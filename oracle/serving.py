"""Oracle of the serving calls (include/pkv.h, "Serving from a paged cache"):
rows quantised into a paged cache, read back, turned to their positions,
attention over it, the weight its tokens receive, and a cache without the
tokens that receive least.

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


def rotate(x, where, offset, freq, interleaved, amplitude):
    """Rows ``x`` (fp64 [tokens][heads][D]) turned to their positions, pair j by (position + offset[sequence]) * freq[j];
    rows without a position as they are."""
    out = x.copy()
    n = 2 * len(freq)
    first, second = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    for i, (s, pos, _, _) in enumerate(where):
        if s < 0 or pos < 0:
            continue
        angle = (float(pos + int(offset[s])) * np.asarray(freq, np.float64)).astype(np.longdouble)
        c, sn = amplitude * np.cos(angle), amplitude * np.sin(angle)
        a, b = x[i][:, first], x[i][:, second]
        out[i][:, first] = a * c - b * sn
        out[i][:, second] = a * sn + b * c
    return out


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


def weigh(cache, tag, page, dtype, where, kv_lens, page_table, pool_pages, q_bits, lse, heads, scale, window, sinks):
    """The attention weight that each cached token receives, fp64 [S][H][max kv_lens], for rows' log-sum-exp ``lse`` (fp32
    [tokens][Hq]); and what error bounds need, of the same shape: the sum of each exponential times scale * (sum |q| (|k -
    zero| + |zero|)) + |score| + |lse|, and the number of exponentials."""
    q = cache_values(q_bits, dtype)
    group = q.shape[1] // heads
    shape = (len(kv_lens), heads, max(1, int(max(kv_lens))))
    out, slack, terms = np.zeros(shape), np.zeros(shape), np.zeros(shape)
    for s in range(len(kv_lens)):
        mine = [(i, pos) for i, (at, pos, _, _) in enumerate(where) if at == s]
        tok = [(t, int(page_table[s, t // page])) for t in range(int(kv_lens[s])) if t // page < page_table.shape[1]]
        tok = [(t, p) for t, p in tok if 0 <= p < pool_pages]
        if not mine or not tok:
            continue
        t_all = np.array([t for t, _ in tok])
        for h in range(heads):
            rows = [row(cache, tag, page, dtype, 0, p, t % page, h) for t, p in tok]
            k, wide = np.stack([r[0] for r in rows]), np.stack([r[1] + r[2] for r in rows])
            for i, pos in mine:
                sees = (t_all <= pos) & ((pos - t_all < window) | (t_all < sinks) if window else True)
                for g in range(h * group, (h + 1) * group):
                    if lse[i, g] == -np.inf or not sees.any():
                        continue
                    score = scale * (k[sees] @ q[i, g])
                    p = np.exp(score - float(lse[i, g]))
                    out[s, h, t_all[sees]] += p
                    reach = scale * (wide[sees] @ np.abs(q[i, g]))
                    slack[s, h, t_all[sees]] += p * (reach + np.abs(score) + abs(float(lse[i, g])))
                    terms[s, h, t_all[sees]] += 1
    return out, slack, terms


def keep(weights, kv_lens, budgets, sinks, recent):
    """Which tokens stay: for each sequence and head of ``weights`` [S][heads][tokens] a list of indices, ascending."""
    out = []
    for w, n, budget in zip(weights, kv_lens, budgets):
        n, rows = int(n), []
        m = min(n, max(0, int(budget)))
        first = min(sinks, m)
        last = min(recent, m - first)
        for x in w:
            key = [(0, 0.0) if np.isnan(v) else (1, float(v)) for v in x[:n]]
            between = sorted(range(first, n - last), key=lambda t: ((-key[t][0], -key[t][1]), t))[:m - first - last]
            rows.append(list(range(first)) + sorted(between) + list(range(n - last, n)))
        out.append(rows)
    return out


def evict(cache, tag, page, kept, kv_lens, table, to_table, weights=None):
    """Rows that stay, moved: ``kept`` as of :func:`keep`, one list for all heads or one for each.  New copies of the cache
    and the weights."""
    pool = (cache["kv"][0] if tag == TAG_FP16 else cache["codes"]).shape[0]
    new = {k: ([a.copy() for a in v] if isinstance(v, list) else v.copy()) for k, v in cache.items()}
    moved = None if weights is None else weights.copy()

    def place(t, s, j):
        p = int(t[s, j // page]) if 0 <= j // page < t.shape[1] else -1
        return (p, j % page) if 0 <= p < pool else None

    heads = cache["kv"][0].shape[2] if tag == TAG_FP16 else cache["codes"].shape[1]
    for s, rows in enumerate(kept):
        for h in range(heads):
            for j, t in enumerate(rows[h if len(rows) > 1 else 0]):
                a, b = place(table, s, t), place(to_table, s, j)
                if a is None or b is None or (to_table is table and t == j):
                    continue
                if tag == TAG_FP16:
                    for w in range(2):
                        new["kv"][w][b[0], b[1], h] = cache["kv"][w][a[0], a[1], h]
                    continue
                size = cache["codes"].shape[2]
                dim = size * 8 // (page * (KEY_BITS[tag] + VALUE_BITS[tag]))
                for w in range(2):
                    lo, hi = tile_bounds(tag, page, dim, w)
                    new["codes"][b[0], h, lo:hi].reshape(page, -1)[b[1]] = \
                        cache["codes"][a[0], h, lo:hi].reshape(page, -1)[a[1]]
                    new["scales"][b[0], h, w, b[1]] = cache["scales"][a[0], h, w, a[1]]
        if moved is not None:
            for h, row_ in enumerate(rows):
                n = int(kv_lens[s])
                moved[s, h, :len(row_)] = weights[s, h, row_]
                moved[s, h, len(row_):n] = 0.0
    return new, moved
