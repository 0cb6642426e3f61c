"""Cases of rotary positions and of eviction: what a program does around the attention over a paged cache.

* ``rotate``  rows turned to their positions: pair j of a row at position p by the angle p * f_j;
* ``append``  queries and keys turned, the keys rounded and written into the cache with the values; read back;
* ``weigh``   the attention weight that cached tokens receive from a call's rows, given the rows' log-sum-exp,
  added to what they had before: out = decay * weights + sum over rows and query heads of exp(scale * q . k - lse);
* ``keep``    which tokens stay under a budget: the first ``sinks``, the last ``recent``, and of the others
  those of the largest weight, equal ones lowest index first; ascending, -1 behind the last;
* ``evict``   the rows that stay moved to the front of their sequence (in place, or to pages of their own), their
  weights with them; the weights behind the last are 0.

Fields of a case: ``heads`` KV heads, ``group`` query heads per KV head, ``dim`` channels per head, ``page`` slots per
page, ``dtype`` (queries, rows, 16-bit pages), ``tag`` (what the cache holds: FP16 = 16-bit rows, else the bits of
keys and values), ``paired`` (16-bit pages hold K slots, then V slots), ``kv`` (tokens of each sequence in the cache, the
new ones included), ``new`` (new tokens of each, dealt in turn), ``scattered`` (the new tokens sit at random places),
``window`` (0: all) and ``sinks``, ``interleaved`` (pairs (2j, 2j + 1), else (j, j + rotary / 2)), ``rotary`` channels that
turn, ``scaling`` of the frequencies and ``amplitude`` of the turned pairs for long contexts, ``far`` (positions start
that far on, as after eviction), ``joint`` (one weight a token, else one for each KV head), ``decay``, ``budget`` (tokens
kept at most), ``ragged`` (a budget for each sequence below that), ``recent``, ``moved`` (evict to other pages).

Codes: [pages][heads][K: page x dim | V: page x dim], two 4-bit codes to a byte, the even channel low.  Scales:
[pages][heads][K, V][page][scale, zero]; a row (one token, one head) stands for code * scale + zero.
"""
import math

import torch

own = False

BITS = {"FP16": (16, 16), "K8V8": (8, 8), "K8V4": (8, 4), "K4V4": (4, 4)}
TAGS = ("FP16", "K8V8", "K8V4", "K4V4")
THETA = 500000.0


def _case(name, op, kv, new="1", tag="K4V4", heads=8, group=4, dim=128, page=16, dtype="bfloat16", paired=False,
          scattered=False, window=0, sinks=0, interleaved=False, rotary=0, scaling="none", amplitude=1.0, far=0,
          joint=True, decay=1.0, budget=0, ragged=False, recent=0, moved=False):
    return {"name": name, "op": op, "tag": tag, "heads": heads, "group": group, "dim": dim, "page": page,
            "dtype": dtype, "paired": paired, "kv": kv, "new": new, "scattered": scattered, "window": window,
            "sinks": sinks, "interleaved": interleaved, "rotary": rotary or dim, "scaling": scaling,
            "amplitude": amplitude, "far": far, "joint": joint, "decay": decay, "budget": budget, "ragged": ragged,
            "recent": recent, "moved": moved}


# The sequences of one decode batch: lengths as a serving program has them in flight, a free slot (0) among them.
BATCH = ("16384,9001,512,15873,4096,1,7777,12288,300,16001,2048,10240,33,14000,6143,8192,0,11111,5000,16384,"
         "900,13579,3000,15000,7200,1025,9999,16200,64,12000,4500,16384")


def listed():
    return [
        # The queries of one decode step, after evictions, so at positions past the cache's slots.
        _case("rotate_step", "rotate", BATCH, far=100000),
        # Queries of a prompt, half of each head turned in interleaved pairs, frequencies and amplitude for long contexts.
        _case("rotate_prompt", "rotate", "32768,5001", "28000,4999", dtype="float16", interleaved=True, rotary=64,
              scaling="wavelength", amplitude=1.2079),
        # One decode step's rows: turned, and the keys and values into a 4-bit cache.
        _case("append_step", "append", BATCH, far=100000),
        # A prompt as long as the 8B-shaped one-layer workload's suffix, keys in 8 bits, values in 4.
        _case("append_prompt", "append", "8192", "8192", tag="K8V4", dtype="float16", scaling="linear"),
        # The weights of the smallest decode step: one sequence of a small model.
        _case("weigh_small", "weigh", "777", heads=2, dim=64, dtype="float16"),
        # A decode step of 32 sequences, ragged, 4-bit cache, weights that fade.
        _case("weigh_step", "weigh", BATCH, decay=0.9),
        # The last rows of long prompts weigh the whole context, each KV head for itself, over 16-bit pages.
        _case("weigh_observe", "weigh", "65536,20011", "32", tag="FP16", joint=False, decay=0.0),
        # Every row of a prompt weighs what it sees.
        _case("weigh_prompt", "weigh", "8192", "8192", tag="FP16", paired=True, joint=False, decay=0.0),
        # What 32 sequences keep, one choice for all heads.
        _case("keep_step", "keep", BATCH, budget=2048, sinks=4, recent=256),
        # What long prompts keep, each KV head for itself, a budget for each prompt.
        _case("keep_long", "keep", "131072,40001", joint=False, budget=16384, ragged=True, sinks=4, recent=32),
        # 32 sequences of a 4-bit cache cut back to their budget in place.
        _case("evict_step", "evict", BATCH, budget=2048, sinks=4, recent=256),
        # Long prompts in 16 bits cut back, each KV head for itself, to pages of their own (the prompt's are shared).
        _case("evict_long", "evict", "65536,20011", tag="FP16", joint=False, budget=16384, ragged=True, sinks=4,
              recent=32, moved=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotate", "append", "weigh", "weigh", "keep", "evict"))
    heads, dim = rng.choice((1, 2, 4, 8, 8)), rng.choice((64, 128, 128, 256))
    group, page = rng.choice((1, 2, 4, 5, 8)), rng.choice((1, 8, 16, 16, 32, 64))
    c = {"heads": heads, "group": group, "dim": dim, "page": page, "dtype": rng.choice(("float16", "bfloat16")),
         "tag": rng.choice(TAGS), "paired": rng.random() < 0.5}
    seqs, new = _log_int(rng, 1, 48), "1"
    most = {"rotate": 33000, "append": 40000, "weigh": 240000, "keep": 1000000, "evict": 85000}[op]
    wide = {"rotate": heads * dim * group / 4, "keep": 1024 * (heads if rng.random() < 0.5 else 1)}.get(op, heads * dim)
    top = max(1, min(131072, int(most * 1024 / (wide * seqs))))
    if op == "append":
        top = max(1, min(top, int(10000 * 4096 / (wide * group * seqs)) + 4))
    kv = [_log_int(rng, max(1, top // 40), top) for _ in range(seqs)]
    c["joint"] = wide == 1024 if op == "keep" else rng.random() < 0.5
    if op in ("rotate", "append"):
        c["interleaved"], c["rotary"] = rng.random() < 0.4, rng.choice((dim, dim, dim // 2, dim // 4, 16))
        c["scaling"] = rng.choice(("none", "linear", "wavelength"))
        c["amplitude"] = 1.0 if c["scaling"] == "none" else round(rng.uniform(1.0, 1.4), 4)
        c["far"] = rng.choice((0, _log_int(rng, 1, 1000000)))
        new = [1 for _ in kv] if rng.random() < 0.4 else [max(1, int(n * rng.uniform(0.2, 1.0))) for n in kv]
        c["scattered"] = rng.random() < 0.3
    elif op == "weigh":
        if rng.random() < 0.4:
            c["window"], c["sinks"] = _log_int(rng, 32, 4096), rng.choice((0, 1, 4, 17, 64))
        c["decay"] = rng.choice((0.0, 1.0, round(rng.uniform(0.5, 1.0), 3)))
        if rng.random() < 0.5:
            kind = rng.randint(1, 4)  # tokens of a decode step; more than one where drafts are checked
            new = [min(kind, n) for n in kv]
        else:
            # a chunk: its score matrix (padded to the longest sequence) stays below the largest listed one
            rows = max(1, int(1.5e9 * min(1, 128 / dim) / (seqs * heads * group * max(kv))))
            new = [min(n, _log_int(rng, max(1, rows // 4), max(1, rows)), 8192) for n in kv]
            c["scattered"] = rng.random() < 0.3
    else:
        c["sinks"], c["recent"] = rng.choice((0, 1, 4, 17, 64)), _log_int(rng, 1, 512)
        c["budget"] = _log_int(rng, max(1, max(kv) // 64), max(kv))
        c["ragged"], c["moved"] = rng.random() < 0.5, op == "evict" and rng.random() < 0.5
    text = lambda v: ",".join(str(n) for n in v)  # noqa: E731
    c = _case("", op, text(kv), new if isinstance(new, str) else text(new), **c)
    del c["name"]
    return c


def _lengths(case):
    kv = [int(n) for n in case["kv"].split(",")]
    new = [int(n) for n in case["new"].split(",")]
    return kv, [min(new[i % len(new)], max(1, n)) for i, n in enumerate(kv)]


def _budgets(case):
    """Most tokens that each sequence keeps."""
    kv, _ = _lengths(case)
    return [max(1, case["budget"] * (3 + i % 5) // 7) if case["ragged"] else case["budget"] for i in range(len(kv))]


def _frequencies(case):
    """The angle that each pair turns by from one position to the next."""
    n = case["rotary"]
    f = [THETA ** (-2.0 * j / n) for j in range(n // 2)]
    if case["scaling"] == "linear":
        return [x / 4.0 for x in f]
    if case["scaling"] == "wavelength":  # short wavelengths as they are, long ones eight times longer, a ramp between
        ramp = [min(1.0, max(0.0, (8192.0 * x / (2.0 * math.pi) - 1.0) / 3.0)) for x in f]
        return [x * (r + (1.0 - r) / 8.0) for x, r in zip(f, ramp)]
    return f


# ---- the plain form: elementary operations in 32 bits; rotations in 64, whose keys lie next to the codes' borders ----

def _next16(h, up):
    """The neighbouring binary16 value of each element."""
    b = h.view(torch.int16).to(torch.int32) & 0xFFFF
    away = (b >= 0x8000) != up
    b = torch.where(b & 0x7FFF == 0, torch.full_like(b, 1 if up else 0x8001), torch.where(away, b + 1, b - 1))
    return torch.where(b >= 0x8000, b - 0x10000, b).to(torch.int16).view(torch.float16)


def _quantise(x, bits):
    """Rows [..., dim] -> (codes uint8 [..., dim], binary16 [..., 2] scale and zero)."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True) + 0.0, x.amax(-1, keepdim=True)
    zero = lo.half()
    zero = torch.where(zero.float() > lo, _next16(zero, False), zero)
    # (the least binary16 that reaches the largest value: decided in 64 bits)
    span = (hi.double() - zero.double() + 0.0) / torch.full_like(hi, 2 ** bits - 1)
    scale = span.float().half()
    scale = torch.where(scale.double() < span, _next16(scale, True), scale)
    s = scale.double()
    codes = torch.where(s > 0, torch.round((x.double() - zero.double()) / s.clamp(min=1e-30)), 0.0)
    return codes.clamp(0, 2 ** bits - 1).to(torch.uint8), torch.cat([scale, zero], -1)


def _pack(codes, bits):
    return codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def _decode(packed, scales, bits, dim):
    c = packed if bits == 8 else torch.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], dim)
    return c.float() * scales[..., :1].float() + scales[..., 1:].float()


def _tiles(st):
    """The K and the V codes of the pool, each [pages][heads][page][bytes of a row]."""
    kb, vb = (st["page"] * st["dim"] * b // 8 for b in BITS[st["tag"]])
    pages, heads = st["codes"].shape[:2]
    return (st["codes"][..., :kb].view(pages, heads, st["page"], -1),
            st["codes"][..., kb:kb + vb].view(pages, heads, st["page"], -1))


def _rows(st):
    """(sequence, position, physical page, slot, whether there is such a row) of every new token."""
    n = st["tokens"]
    at = torch.arange(n, device=st["kv_lens"].device)
    seq = torch.bucketize(at, st["token_start"][1:].long(), right=True)
    if st["positions"] is None:
        pos = st["kv_lens"].long()[seq] - st["token_start"].long()[seq + 1] + at
    else:
        pos = st["positions"].long()
    page = st["page_table"].long()[seq, pos.clamp(min=0) // st["page"]]
    return seq, pos, page.clamp(min=0), pos.clamp(min=0) % st["page"], (pos >= 0) & (page >= 0)


def _plain_rotate(st, x, seq, pos):
    """Rows [tokens, heads, dim] turned; a row without a position stays as it is."""
    turn = (pos + st["offset"].long()[seq]).double()[:, None] * st["inv_freq"].to(pos.device)
    turn = torch.where((pos >= 0)[:, None], turn, 0.0)
    gain = torch.where(pos >= 0, st["amplitude"], 1.0)[:, None]
    cos, sin = (torch.cos(turn) * gain)[:, None], (torch.sin(turn) * gain)[:, None]
    n, y = st["rotary"], x.double()
    first, second = (slice(0, n, 2), slice(1, n, 2)) if st["interleaved"] else (slice(0, n // 2), slice(n // 2, n))
    out = y.clone()
    out[..., first] = y[..., first] * cos - y[..., second] * sin
    out[..., second] = y[..., first] * sin + y[..., second] * cos
    return out.float().to(x.dtype)


def _plain_append(st):
    seq, pos, page, slot, there = _rows(st)
    page = torch.where(there, page, st["pool"] - 1)  # rows without a place: a page of the pool that nobody owns
    k = _plain_rotate(st, st["k"], seq, pos)
    back = []
    for which, x in enumerate((k, st["v"])):
        bits = BITS[st["tag"]][which]
        if bits == 16:
            cache = (st["k_cache"], st["v_cache"])[which]
            cache[page, slot] = x
            got = cache[page, slot]
        else:
            codes, scales = _quantise(x, bits)
            tile = _tiles(st)[which]
            tile[page, :, slot] = _pack(codes, bits)
            st["scales"][page, :, which, slot] = scales
            got = _decode(tile[page, :, slot], st["scales"][page, :, which, slot], bits, st["dim"]).to(x.dtype)
        back.append(torch.where(there[:, None, None], got, 0.0))
    return [_plain_rotate(st, st["q"], seq, pos), *back]


def _plain_scores(st):
    """Masked scores [seqs, heads, new tokens padded to the most, group, tokens], and each one's row of the call."""
    heads, group, dim, page, most = st["heads"], st["group"], st["dim"], st["page"], st["most_new"]
    _, pos, _, _, _ = _rows(st)
    seqs, dev = st["kv_lens"].numel(), pos.device
    tok = torch.arange(st["most_kv"], device=dev).expand(seqs, -1)
    there = tok < st["kv_lens"].long()[:, None]
    phys = st["page_table"].long().gather(1, (tok // page).clamp(max=st["page_table"].shape[1] - 1))
    there, phys, slot = there & (phys >= 0), phys.clamp(min=0), tok % page
    if st["tag"] == "FP16":
        k = st["k_cache"][phys, slot].float()
    else:
        k = _decode(_tiles(st)[0][phys, :, slot], st["scales"][phys, :, 0, slot], BITS[st["tag"]][0], dim)
    k = k.masked_fill_(~there[:, :, None, None], 0.0).permute(0, 2, 3, 1).contiguous()  # [seqs, heads, dim, tokens]
    j = torch.arange(most, device=dev)
    row = st["token_start"][:-1].long()[:, None] + j
    mine = row < st["token_start"][1:].long()[:, None]
    row = row.clamp(max=st["tokens"] - 1)
    q = st["q"].float()[row].view(seqs, most, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(seqs, heads, -1, dim)
    s = torch.matmul(q, k).mul_(dim ** -0.5).view(seqs, heads, most, group, -1)
    at = pos[row][:, :, None]
    sees = mine[:, :, None] & there[:, None, :] & (tok[:, None, :] <= at)
    if st["window"]:
        sees = sees & ((tok[:, None, :] > at - st["window"]) | (tok[:, None, :] < st["sinks"]))
    return s.masked_fill_(~sees[:, None, :, None, :], -math.inf), row, mine


def _plain_weigh(st):
    s, row, mine = _plain_scores(st)
    seqs, heads, most, group, tokens = s.shape
    lse = st["lse"][row].view(seqs, most, heads, group).permute(0, 2, 1, 3)[..., None]
    got = s.sub_(torch.where(lse == -math.inf, math.inf, lse)).exp_().sum((2, 3))
    if st["joint"]:
        got = got.sum(1, keepdim=True)
    if st["decay"]:
        got = got + st["weights"] * st["decay"]
    here = torch.arange(tokens, device=s.device) < st["kv_lens"].long()[:, None, None]
    st["out"].copy_(torch.where(here, got, st["out"]))
    return st["out"]


def _plain_keep(st):
    w, n = st["weights"], st["kv_lens"].long()[:, None, None]
    t = torch.arange(w.shape[2], device=w.device)
    m = torch.minimum(n, st["budgets"].long()[:, None, None])
    first = torch.minimum(m, torch.full_like(m, st["sinks"]))
    last = torch.minimum(m - first, torch.full_like(m, st["recent"]))
    key = torch.where((t < first) | ((t >= n - last) & (t < n)), math.inf, torch.where(t < n, w, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :st["budget"]]
    j = torch.arange(order.shape[2], device=w.device)
    order = torch.sort(torch.where(j < m, order, w.shape[2])).values
    order = torch.where(j < m, order, -1).int()
    return [torch.nn.functional.pad(order, (0, st["budget"] - order.shape[2]), value=-1), m[:, 0, 0].int()]


def _plain_evict(st):
    kept, page, heads = st["kept"].long(), st["page"], st["heads"]
    seqs, dev = kept.shape[0], kept.device
    m = st["kept_lens"].long()[:, None, None]
    j = torch.arange(kept.shape[2], device=dev).expand_as(kept)
    on = j < m
    seq = torch.arange(seqs, device=dev)[:, None, None]
    at = kept.clamp(min=0)
    source = st["page_table"].long()[seq, at // page]
    table = st["other_table"] if st["moved"] else st["page_table"]
    target = table.long()[seq, (j // page).clamp(max=table.shape[1] - 1)]
    target = torch.where(on, target, st["pool"] - 1)  # (a page of the pool that nobody owns)
    source, slot = source.clamp(min=0).expand(-1, heads, -1), (at % page).expand(-1, heads, -1)
    target, to = target.expand(-1, heads, -1), (j % page).expand(-1, heads, -1)
    head = torch.arange(heads, device=dev)[None, :, None]
    if st["tag"] == "FP16":
        for cache in (st["k_cache"], st["v_cache"]):
            cache[target, to, head] = cache[source, slot, head]
        out = [st["k_cache"][:-1], st["v_cache"][:-1]]
    else:
        for tile in _tiles(st):
            tile[target, head, to] = tile[source, head, slot]
        scales = st["scales"].permute(0, 1, 3, 2, 4)
        scales[target, head, to] = scales[source, head, slot]
        out = [st["codes"][:-1], st["scales"][:-1]]
    w, t = st["weights"], torch.arange(st["weights"].shape[2], device=dev)
    moved = torch.nn.functional.pad(torch.where(on, w.gather(2, at), 0.0), (0, max(0, t.numel() - kept.shape[2])))
    w.copy_(torch.where(t < st["kv_lens"].long()[:, None, None], moved[..., :t.numel()], w))
    return out + [w]


# ---- states ----

def _values(gen, shape, dim, dev):
    """Rows as the path meets them: N(0, 1), one rotary pair of channels of each head scaled by 8."""
    x = torch.randn(shape, generator=gen, device=dev)
    pair = torch.randint(0, dim // 2, (shape[-2],), generator=gen, device=dev)
    head = torch.arange(shape[-2], device=dev)
    gain = torch.ones(shape[-2:], device=dev)
    gain[head, pair] = 8.0
    gain[head, pair + dim // 2] = 8.0
    return x.mul_(gain)


def _weights(gen, shape, dev):
    """Accumulated weights: a long tail, as attention leaves them, some equal and some tokens never seen."""
    w = torch.randn(shape, generator=gen, device=dev).mul_(2.0).exp_()
    coarse = torch.rand(shape, generator=gen, device=dev)
    w = torch.where(coarse < 0.3, (w * 16.0).round() / 16.0, w)
    return torch.where(coarse > 0.95, 0.0, w)


def prepare(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    kv, new = _lengths(case)
    heads, dim, page, bits, op = case["heads"], case["dim"], case["page"], BITS[case["tag"]], case["op"]
    st = {k: v for k, v in case.items() if k not in ("kv", "new", "name")}
    st |= {"tokens": sum(new), "most_new": max(new), "most_kv": max(kv)}
    need = [-(-n // page) for n in kv]
    other = [-(-min(n, b) // page) if case["moved"] else 0 for n, b in zip(kv, _budgets(case))]
    st["pool"] = pool = sum(need) + sum(other) + max(2, sum(need) // 8)
    order = torch.randperm(pool - 1, generator=gen, device=dev).int()  # the last page belongs to nobody

    def table(need, first):
        begin = torch.tensor([0] + need).cumsum(0)[:-1].to(dev) + first
        at = torch.arange(max(1, max(need)), device=dev).expand(len(need), -1)
        owned = at < torch.tensor(need, device=dev)[:, None]
        return torch.where(owned, order[(begin[:, None] + at).clamp(max=pool - 2)], -1).int().contiguous()

    st["page_table"] = table(need, 0)
    if case["moved"]:
        st["other_table"] = table(other, sum(need))
    st["kv_lens"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    st["token_start"] = torch.tensor([0] + new).cumsum(0).int().to(dev)
    st["positions"] = None
    if case["scattered"]:
        st["positions"] = torch.cat([torch.randperm(k, generator=gen, device=dev)[:n].sort().values if k else
                                     torch.full((n,), -1, device=dev) for k, n in zip(kv, new)]).int()
    if op in ("rotate", "append"):
        st["inv_freq"] = torch.tensor(_frequencies(case), dtype=torch.float64)
        st["offset"] = (torch.rand(len(kv), generator=gen, device=dev) * (case["far"] + 1)).int()
    if op in ("rotate", "append", "weigh"):
        st["q"] = torch.randn((sum(new), heads * case["group"], dim), generator=gen, device=dev).to(dtype)
    if op == "append":
        st |= {"k": _values(gen, (sum(new), heads, dim), dim, dev).to(dtype),
               "v": _values(gen, (sum(new), heads, dim), dim, dev).to(dtype)}
    if op in ("rotate", "keep"):
        st["pool"] = pool = 1  # (neither looks at what the cache holds)
    if case["tag"] == "FP16":
        # paired: one buffer [pages][K, V][page][heads][dim]; else two of [pages][page][heads][dim]
        k, v = (_values(gen, (pool, page, heads, dim), dim, dev).to(dtype) for _ in range(2))
        if case["paired"]:
            both = torch.stack([k, v], 1)
            k, v = both[:, 0], both[:, 1]
        st |= {"k_cache": k, "v_cache": v}
    elif op == "append":
        st["codes"] = torch.zeros((pool, heads, page * dim * sum(bits) // 8), dtype=torch.uint8, device=dev)
        st["scales"] = torch.zeros((pool, heads, 2, page, 2), dtype=torch.float16, device=dev)
    else:
        codes, scales = [], []
        for b in bits:
            c, s = _quantise(_values(gen, (pool, page, heads, dim), dim, dev).to(dtype), b)
            codes.append(_pack(c, b).permute(0, 2, 1, 3).reshape(pool, heads, -1))
            scales.append(s.permute(0, 2, 1, 3))
            del c, s
        st |= {"codes": torch.cat(codes, -1).contiguous(), "scales": torch.stack(scales, 2).contiguous()}
    if op in ("weigh", "keep", "evict"):
        st["weights"] = _weights(gen, (len(kv), 1 if case["joint"] else heads, max(kv)), dev)
    if op == "weigh":
        st["out"] = torch.zeros_like(st["weights"])
        s, row, mine = _plain_scores(st)
        top = s.amax(-1, keepdim=True)
        lse = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_().sum(-1).log_() + top[..., 0]
        lse = lse.permute(0, 2, 1, 3).reshape(len(kv), max(new), -1)
        st["lse"] = lse[mine].contiguous()
    if op in ("keep", "evict"):
        st["budgets"] = torch.tensor(_budgets(case), dtype=torch.int32, device=dev)
    if op == "evict":
        st["kept"], st["kept_lens"] = _plain_keep(st)
    return st


def _handles(st):
    """What a serving program keeps beside the tensors: the cache and the batch, described once."""
    if "cache" not in st:
        from paper_2609_26219_amd import serving
        rope = {}
        if "inv_freq" in st:
            rope = {"rope_style": int(st["interleaved"]), "rotary_dim": st["rotary"],
                    "inv_freq": st["inv_freq"].tolist(), "rope_amplitude": st["amplitude"]}
        st["cache"] = serving.PagedCache(
            num_kv_heads=st["heads"], head_dim=st["dim"], page_size=st["page"], dtype=getattr(torch, st["dtype"]),
            tag=TAGS.index(st["tag"]), codes=st.get("codes"), scales=st.get("scales"), k_cache=st.get("k_cache"),
            v_cache=st.get("v_cache"), **rope)
        st["batch"] = serving.Batch(token_start=st["token_start"], kv_lens=st["kv_lens"], page_table=st["page_table"],
                                    positions=st["positions"], num_tokens=st["tokens"], max_tokens=st["most_new"],
                                    max_kv_len=st["most_kv"])
    return st["cache"], st["batch"]


def run(st):
    op = st["op"]
    if not own:
        if op == "rotate":
            seq, pos, _, _, _ = _rows(st)
            return _plain_rotate(st, st["q"], seq, pos)
        return {"append": _plain_append, "weigh": _plain_weigh, "keep": _plain_keep, "evict": _plain_evict}[op](st)
    from paper_2609_26219_amd import serving
    cache, batch = _handles(st)
    if op == "rotate":
        return serving.rotate(cache, batch, st["q"], position_offset=st["offset"])
    if op == "append":
        q = serving.append_rotated(cache, batch, st["q"], st["k"], st["v"], position_offset=st["offset"])
        return [q, *serving.read(cache, batch)]
    if op == "weigh":
        return serving.attention_weights(cache, batch, st["q"], st["lse"], st["out"], weights=st["weights"],
                                         decay=st["decay"], window=st["window"], sinks=st["sinks"])
    if op == "keep":
        return list(serving.keep(cache, batch, st["weights"], st["budget"], sinks=st["sinks"], recent=st["recent"],
                                 budgets=st["budgets"] if st["ragged"] else None))
    serving.evict(cache, batch, st["kept"], st["kept_lens"], weights=st["weights"],
                  page_table=st["other_table"] if st["moved"] else None)
    # (codes are returned as they lie: the operator moves them as bytes, and they come out equal or wrong)
    held = ("k_cache", "v_cache") if st["tag"] == "FP16" else ("codes", "scales")
    return [st[h][:-1] for h in held] + [st["weights"]]


def _visible(case):
    """For each sequence: (visible tokens summed over its new rows, tokens that some row sees)."""
    kv, new = _lengths(case)
    w, s, got = case["window"], case["sinks"], []
    for k, n in zip(kv, new):
        n = min(n, k)
        if case["scattered"]:  # random places: the mean over them
            mean = (k + 1) / 2 if not w else min(w + s, (k + 1) / 2)
            got.append((n * mean, k if not w else min(k, s + n * w)))
        elif not w:
            got.append((n * (k - n) + n * (n + 1) // 2, k))
        else:
            got.append((sum(min(t + 1, w + min(s, max(0, t + 1 - w))) for t in range(k - n, k)),
                        min(k, w + n - 1 + s) if n else 0))
    return got


def work(case):
    kv, new = _lengths(case)
    op, heads, dim, group = case["op"], case["heads"], case["dim"], case["group"]
    rows = sum(min(n, k) for k, n in zip(kv, new))
    weights = 4 * (1 if case["joint"] else heads) * sum(kv)
    half16 = heads * dim * 2
    half = [half16 if b == 16 else heads * (dim * b // 8 + 4) for b in BITS[case["tag"]]]
    if op == "rotate":
        return {"bytes": 2 * rows * group * half16, "flops": 3.0 * rows * heads * group * case["rotary"]}
    if op == "append":  # rows in, queries and codes out; codes in, rows out
        return {"bytes": rows * (2 * group * half16 + 2 * 2 * half16 + 2 * sum(half)),
                "flops": rows * heads * (3.0 * (group + 1) * case["rotary"] + 16.0 * dim)}
    if op == "weigh":
        seen = _visible(case)
        return {"bytes": sum(t for _, t in seen) * half[0] + rows * heads * group * (2 * dim + 4) +
                weights * (2 if case["decay"] else 1),
                "flops": 2.0 * heads * group * dim * sum(p for p, _ in seen)}
    keep = sum(min(n, b) for n, b in zip(kv, _budgets(case)))
    index = 4 * (1 if case["joint"] else heads) * keep
    if op == "keep":
        return {"bytes": weights + index, "flops": weights / 4.0}
    stay = 0  # the tokens that evict leaves where they are, at least: the sinks, and sequences within their budget
    if not case["moved"]:
        stay = sum(n if n <= b else min(case["sinks"], b) for n, b in zip(kv, _budgets(case)))
    return {"bytes": 2 * (keep - stay) * sum(half) + index + 4 * (1 if case["joint"] else heads) * keep + weights,
            "flops": 1.0}


# ---- the definition in 64 bits ----

def _exact16(x, up):
    """The nearest binary16 value of doubles that is not below (up) or not above them."""
    h = x.to(torch.float16)
    step = _next16(h, up).double()
    return torch.where((h.double() < x) if up else (h.double() > x), step, h.double())


def _exact_rows(x, bits):
    """What rows [..., dim] stand for once they are held in so many bits."""
    x = x.double()
    if bits == 16:
        return x
    zero = _exact16(x.amin(-1, keepdim=True), False)
    scale = _exact16((x.amax(-1, keepdim=True) - zero) / torch.full_like(zero, 2 ** bits - 1), True)
    codes = torch.round((x - zero) / torch.where(scale > 0, scale, 1.0)).clamp(0, 2 ** bits - 1)
    return torch.where(scale > 0, codes * scale, 0.0) + zero


def _exact_turned(case, x, at):
    """One sequence's rows as complex numbers, turned."""
    n, x = case["rotary"], x.double()
    pairs = x[..., :n].reshape(*x.shape[:-1], n // 2, 2) if case["interleaved"] else \
        torch.stack([x[..., :n // 2], x[..., n // 2:n]], -1)
    f = torch.tensor(_frequencies(case), dtype=torch.float64, device=x.device)
    by = torch.polar(torch.full((), case["amplitude"], dtype=torch.float64, device=x.device), at.double()[:, None] * f)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by[:, None, :])
    y = y.reshape(*x.shape[:-1], n) if case["interleaved"] else torch.cat([y[..., 0], y[..., 1]], -1)
    return torch.cat([y, x[..., n:]], -1)


def exact(case, seed):
    op = case["op"]
    if op == "keep":
        return None  # whole numbers
    st = prepare(case, seed)
    kv, new = _lengths(case)
    bits, dim, page, heads = BITS[case["tag"]], case["dim"], case["page"], case["heads"]
    dev = st["kv_lens"].device

    def cached(which, phys, slot):
        """Rows [tokens, heads, dim] of the cache as doubles."""
        if case["tag"] == "FP16":
            return st["v_cache" if which else "k_cache"][phys, slot].double()
        start = which * page * dim * bits[0] // 8
        size = page * dim * bits[which] // 8
        raw = st["codes"][:, :, start:start + size].reshape(st["codes"].shape[0], heads, page, -1)[phys, :, slot]
        code = torch.empty(*raw.shape[:-1], dim, dtype=torch.float64, device=dev)
        if bits[which] == 8:
            code.copy_(raw)
        else:
            code[..., 0::2], code[..., 1::2] = raw % 16, raw // 16
        sz = st["scales"][phys, :, which, slot].double()
        return code * sz[..., 0:1] + sz[..., 1:2]

    if op == "evict":
        w = st["weights"].double()
        pair = [c.double() for c in (st["k_cache"], st["v_cache"])] if case["tag"] == "FP16" else [None, None]
        now = [c.clone() if c is not None else None for c in pair]
        scales = None if case["tag"] == "FP16" else st["scales"].double()
        moved = w.clone()
        sc = None if scales is None else scales.clone()
        tables = (st["page_table"], st["other_table"] if case["moved"] else st["page_table"])
        for s, n in enumerate(kv):
            m = int(st["kept_lens"][s])
            moved[s, :, :n] = 0.0
            to = torch.arange(m, device=dev)
            there = tables[1][s].long()[to // page]
            for h in range(heads):
                g = 0 if case["joint"] else h
                at = st["kept"][s, g, :m].long()
                moved[s, g, :m] = w[s, g, at]
                here = tables[0][s].long()[at // page]
                for which in range(2):
                    if scales is None:
                        now[which][there, to % page, h] = pair[which][here, at % page, h]
                    else:
                        sc[there, h, which, to % page] = scales[here, h, which, at % page]
        return [now[0][:-1], now[1][:-1], moved] if scales is None else [None, sc[:-1], moved]

    outs, at = [], 0
    weights = st["out"].double() if op == "weigh" else None
    for s, (k_len, n) in enumerate(zip(kv, new)):
        rows = slice(at, at + n)
        at += n
        pos = st["positions"][rows].long() if case["scattered"] else torch.arange(k_len - n, k_len, device=dev)
        if op in ("rotate", "append"):
            if not k_len:  # no position
                turn = lambda x: x.double()  # noqa: E731
            else:
                turn = lambda x: _exact_turned(case, x, pos + int(st["offset"][s]))  # noqa: E731
            got = [turn(st["q"][rows])]
            if op == "append":
                k = turn(st["k"][rows]).float().to(st["k"].dtype)
                got += [_exact_rows(x, b) if k_len else torch.zeros_like(x, dtype=torch.float64)
                        for x, b in zip((k, st["v"][rows]), bits)]
            outs.append(got)
            continue
        if not k_len:
            continue
        table = st["page_table"][s].long()
        tok = torch.arange(k_len, device=dev)
        k = cached(0, table[tok // page], tok % page)
        total = torch.zeros((heads, k_len), dtype=torch.float64, device=dev)
        step = max(1, int(2.5e8 / k_len))
        for r0 in range(0, n, step):
            p0 = pos[r0:r0 + step]
            ok = tok[None] <= p0[:, None]
            if case["window"]:
                ok &= (p0[:, None] - tok[None] < case["window"]) | (tok[None] < case["sinks"])
            for h in range(heads * case["group"]):
                g = h // case["group"]
                score = st["q"][rows][r0:r0 + step, h].double() @ k[:, g].T.contiguous() / math.sqrt(dim)
                p = torch.exp(score - st["lse"][rows][r0:r0 + step, h].double()[:, None])
                total[g] += torch.where(ok, p, 0.0).sum(0)
        if case["joint"]:
            total = total.sum(0, keepdim=True)
        weights[s, :, :k_len] = total + case["decay"] * st["weights"][s, :, :k_len].double()
    if op == "weigh":
        return weights
    outs = [torch.cat([p[w] for p in outs]) for w in range(len(outs[0]))]
    return outs[0] if op == "rotate" else outs
