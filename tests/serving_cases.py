"""Small seeded cases of the serving calls, on the host, and the oracle's word on them."""
import numpy as np

from oracle import quantize as oq
from oracle import serving as os_
from oracle.restore import output_values, round_to_output

UNIT = {0: 2.0 ** -11, 1: 2.0 ** -8}  # half a unit in the last place, relative: binary16, bfloat16


class Case:
    """Tensors of one call on the host (uint16 bits), the cache among them.

    ``lens`` tokens of each sequence in the cache, ``new`` rows of each in the
    call; ``holes`` unmaps that many owned pages; ``poison`` fills every slot that no
    sequence owns (and slots past a sequence's end) with NaN, or codes with NaN scales."""

    def __init__(self, seed, tag, dtype, H, group, D, P, lens, new, scattered=False, holes=0, layers=1, layer=0,
                 scale_of_values=1.0, poison=True, paired=False, spare_pages=3, wide=0):
        rng = np.random.default_rng(seed)
        self.tag, self.dtype, self.H, self.group, self.D, self.P = tag, dtype, H, group, D, P
        self.layers, self.layer, self.paired = layers, layer, paired
        self.lens = np.array(lens, np.int32)
        need = [-(-n // P) for n in lens]
        self.pool = sum(need) + spare_pages
        order = rng.permutation(self.pool)
        width = max(1, max(need)) + wide
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        new = [new[i % len(new)] for i in range(len(lens))]
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.start[-1])
        self.most_new, self.most_kv = max(new), max(lens)
        self.positions = None
        if scattered:
            self.positions = np.concatenate([rng.permutation(max(n, m))[:m] if n else np.full(m, -1)
                                             for n, m in zip(lens, new)]).astype(np.int32)
        draw = lambda *shape: self.bits(rng.standard_normal(shape) * scale_of_values)  # noqa: E731
        outlier = rng.integers(0, D, H)
        values = [rng.standard_normal((self.pool, P, H, D)) * scale_of_values for _ in range(2)]
        for v in values:
            v[:, :, np.arange(H), outlier] *= 8.0
        nan = {0: 0x7E00, 1: 0x7FC0}[dtype]
        owned = np.zeros((self.pool, P), bool)
        for s, n in enumerate(lens):
            for t in range(n):
                owned[self.table[s, t // P], t % P] = True
        rows = [self.bits(v) for v in values]
        if tag == 0:
            for r in rows:
                if poison:
                    r[~owned] = nan
            self.cache = {"kv": rows}
        else:
            size = P * D * (oq.KEY_BITS[tag] + oq.VALUE_BITS[tag]) // 8
            self.cache = {"codes": rng.integers(0, 256, (self.pool, H, size), dtype=np.uint8),
                          "scales": np.full((self.pool, H, 2, P, 2), 0x7E00, np.uint16)}
            where = [(0, 0, p, s) for p in range(self.pool) for s in range(P) if owned[p, s] or not poison]
            flat = [np.stack([r[p, s] for _, _, p, s in where]) if where else r[:0, 0] for r in rows]
            os_.append(self.cache, tag, P, where, *flat, dtype)
        for _ in range(holes):
            s = int(rng.integers(0, len(lens)))
            if need[s]:
                self.table[s, int(rng.integers(0, need[s]))] = rng.choice([-1, -7, self.pool, 2 ** 31 - 1])
        self.q = draw(self.tokens, H * group, D)
        self.k, self.v = draw(self.tokens, H, D), draw(self.tokens, H, D)

    def bits(self, x):
        return round_to_output(np.asarray(x, np.float64), self.dtype)

    def where(self):
        return os_.places(self.start, self.lens, self.table, self.P, self.pool, self.positions, self.tokens)

    def copy_of_cache(self):
        return {k: ([a.copy() for a in v] if isinstance(v, list) else v.copy()) for k, v in self.cache.items()}

    def attend(self, scale=None, window=0, sinks=0):
        return os_.attend(self.cache, self.tag, self.P, self.dtype, self.where(), self.lens, self.table, self.pool,
                          self.q, self.H, self.D ** -0.5 if scale is None else scale, window, sinks)


def check_read(case, got, which):
    """Rows read back are the definition's, within the double rounding of r18-like windows: half a unit in the last
    place, plus 2^-23 relative for the single-precision step before it, plus half a subnormal step of binary16."""
    for i, (s, pos, phys, slot) in enumerate(case.where()):
        for h in range(case.H):
            if s < 0:
                continue
            want = np.zeros(case.D) if phys < 0 else os_.row(case.cache, case.tag, case.P, case.dtype, which, phys,
                                                             slot, h)[0]
            have = output_values(got[i, h], case.dtype)
            both_nan = np.isnan(want) & np.isnan(have)
            tol = np.abs(want) * (UNIT[case.dtype] * (1 + 2.0 ** -9)) + (2.0 ** -25 if case.dtype == 0 else 0.0)
            assert (both_nan | (np.abs(have - want) <= tol)).all(), (i, h, which)


def check_attention(case, out_bits, lse, window=0, sinks=0, scale=None):
    """Every output element and log-sum-exp within its derived bound.

    An element rounds once to the output type (u). Each probability carries its own rounding u_p to the matrix
    operand's type, on the part of v that goes through it (|v - zero|, zero = the row's value at mid-code), and a
    relative error from its score: single-precision sums of D products, scaled, and the base-2 exponential, together
    4 * delta with delta = 2^-23 * (D / 8 + 16) * reach, and 2^-18 for the exponential's argument and the sums over tokens.  Codes'
    queries are binary16 relative to the row's largest: 2^-25 of it absolute, within the same reach.  Probabilities
    below binary16's range (2^-38 of the largest) are dropped."""
    exact, lse_exact, mass, whole, reach = case.attend(scale, window, sinks)
    have = output_values(out_bits, case.dtype)
    u_p = 2.0 ** -8 if case.tag == 0 and case.dtype == 1 else 2.0 ** -11
    delta = 2.0 ** -23 * (case.D / 8 + 16) * reach
    u = UNIT[case.dtype]
    tol = u * np.abs(exact) * (1 + u) + (u_p * 1.01 + 2.0 ** -24 * case.most_kv) * mass + \
        (4 * delta + 2.0 ** -18)[:, :, None] * whole + (2.0 ** -25 if case.dtype == 0 else 2.0 ** -133)
    off = np.abs(have - exact)
    assert (off <= tol).all(), float((off / tol).max())
    empty = np.isneginf(lse_exact)
    assert (np.isneginf(lse) == empty).all() and not np.isnan(lse).any()
    assert (have[empty] == 0).all()
    d = np.abs(lse[~empty] - lse_exact[~empty])
    assert (d <= 2 * delta[~empty] + 2.0 ** -19 * (1 + np.abs(lse_exact[~empty]))).all(), float(d.max())
