"""Eviction on the GPU against the oracle, all of it bit for bit: which tokens stay under a budget, and the cache and the
weights without the others; and the calls of a bounded cache one after the other, as a decode loop makes them."""
import numpy as np
import pytest

from oracle import serving as os_
from paper_2609_26219_amd import binding as pb
from serving_cases import Case
from test_serving_gpu import _batch, _cache, _down, _state, _up

pytestmark = pytest.mark.gpu

FP16, K8V8, K8V4, K4V4 = range(4)
HALF, BF16 = 0, 1


@pytest.fixture(scope="module")
def torch():
    import torch as _t
    if not _t.cuda.is_available():
        pytest.skip("no GPU")
    pb.load()
    return _t


def _dev(torch, a):
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


def _sequences(torch, lens, heads=1, D=64, P=16):
    """A cache and a batch of which only the lengths are looked at."""
    from paper_2609_26219_amd import serving
    import paper_2609_26219_amd.workloads as wl

    cache = serving.PagedCache(heads, D, P, torch.bfloat16, wl.TAG_K4V4, pool_pages=1)
    width = max(1, -(-max(lens) // P))
    table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    start = torch.zeros(len(lens) + 1, dtype=torch.int32, device="cuda")
    return cache, serving.Batch(start, _dev(torch, lens), table, 0, max_kv_len=max(1, max(lens)))


def _kinds(rng, shape, kind):
    w = rng.exponential(1.0, shape).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 2) / 2
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "zeros":
        w = np.where(rng.random(shape) < 0.5, np.where(rng.random(shape) < 0.5, 0.0, -0.0), w).astype(np.float32)
    elif kind == "signs":
        w = rng.standard_normal(shape).astype(np.float32) * np.float32(10.0) ** rng.integers(-30, 30, shape).astype(np.float32)
    elif kind == "odd":
        w[rng.random(shape) < 0.2] = np.nan
        w[rng.random(shape) < 0.2] = np.inf
        w[rng.random(shape) < 0.2] = -np.inf
        w[rng.random(shape) < 0.2] = np.float32(1e-44)
    elif kind == "close":
        w = (np.float32(1.0) + rng.integers(0, 200, shape).astype(np.float32) * np.float32(2.0 ** -23)).astype(np.float32)
    return w


def _expect(kept, budget, heads, S):
    want = np.full((S, heads, budget), -1, np.int32)
    for s, rows in enumerate(kept):
        for h, r in enumerate(rows):
            want[s, h, :len(r)] = r
    return want


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "zeros", "signs", "odd", "close"])
@pytest.mark.parametrize("lens,heads,budget,sinks,recent", [
    ((100, 1, 0, 37, 2), 1, 20, 4, 8), ((1000, 64, 65), 3, 64, 0, 0), ((5000,), 2, 777, 1, 300),
    ((300, 301), 1, 299, 17, 64), ((40, 50), 1, 5, 9, 9), ((40, 50), 2, 10, 3, 100), ((2049, 1025, 1024), 1, 1000, 0, 1),
])
def test_keep(torch, kind, lens, heads, budget, sinks, recent):
    from paper_2609_26219_amd import serving

    rng = np.random.default_rng(len(kind) + budget)
    cache, batch = _sequences(torch, lens, heads)
    w = _kinds(rng, (len(lens), heads, max(lens)), kind)
    kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), budget, sinks, recent)
    want = os_.keep(w, lens, [budget] * len(lens), sinks, recent)
    assert kept_lens.tolist() == [len(r[0]) for r in want]
    assert np.array_equal(kept.cpu().numpy(), _expect(want, budget, heads, len(lens)))


@pytest.mark.parametrize("n", [32767, 32768, 32769, 40001, 131072])
@pytest.mark.parametrize("kind", ["plain", "zeros", "equal"])
def test_keep_of_long_rows(torch, n, kind):
    """Up to where a row's keys stay in registers, and past it; against a stable sort."""
    from paper_2609_26219_amd import serving

    lens, heads = (n, n // 2, n - 1), 2
    cache, batch = _sequences(torch, lens, heads)
    w = _kinds(np.random.default_rng(n), (3, heads, n), kind)
    for budget, sinks, recent in ((n // 8, 4, 32), (n - 5, 0, 0), (65, 64, 0)):
        kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), budget, sinks, recent)
        got = kept.cpu().numpy()
        for s, length in enumerate(lens):
            m = min(length, budget)
            first = min(sinks, m)
            last = min(recent, m - first)
            for h in range(heads):
                key = w[s, h, first:length - last] + 0.0
                order = np.argsort(-key, kind="stable")[:m - first - last] + first
                want = np.concatenate([np.arange(first), np.sort(order), np.arange(length - last, length)])
                assert np.array_equal(got[s, h, :m], want) and (got[s, h, m:] == -1).all()
        assert kept_lens.tolist() == [min(length, budget) for length in lens]


def test_keep_of_many_long_rows(torch):
    """More rows than are cut into segments: one workgroup each, longer than its registers."""
    from paper_2609_26219_amd import serving

    n, S = 33000, 130
    lens = tuple(n - 7 * s for s in range(S))
    cache, batch = _sequences(torch, lens)
    w = _kinds(np.random.default_rng(3), (S, 1, n), "ties")
    w[5] = 1.0  # more equal ones than LDS lists
    kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), 4000, 3, 50)
    got = kept.cpu().numpy()
    for s in range(0, S, 5):
        order = np.argsort(-w[s, 0, 3:lens[s] - 50], kind="stable")[:4000 - 53] + 3
        want = np.concatenate([np.arange(3), np.sort(order), np.arange(lens[s] - 50, lens[s])])
        assert np.array_equal(got[s, 0], want)
    assert (kept_lens == 4000).all()


def test_keep_on_streams_and_in_graphs(torch):
    """Long rows' workspaces: two streams at once, and two graphs replayed in turn as weights and lengths change."""
    from paper_2609_26219_amd import serving

    n = 50000
    cache, batch = _sequences(torch, (n, n - 9), 2)
    ws = [torch.rand((2, 2, n), device="cuda") for _ in range(2)]
    outs = [tuple(torch.empty_like(t) for t in serving.keep(cache, batch, ws[0], 6000, 4, 9)) for _ in ws]
    want = [serving.keep(cache, batch, w, 6000, 4, 9)[0].clone() for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    torch.cuda.synchronize()
    for _ in range(10):
        for w, out, stream in zip(ws, outs, streams):
            with torch.cuda.stream(stream):
                serving.keep(cache, batch, w, 6000, 4, 9, out=out)
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], x) for o, x in zip(outs, want))
    graphs = []
    for w, out in zip(ws, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            serving.keep(cache, batch, w, 6000, 4, 9, out=out)
        graphs.append(g)
    for i in range(4):
        for w in ws:
            w.copy_(torch.rand_like(w))
        batch.keep[1].sub_(11)
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        for w, out in zip(ws, outs):
            eager = serving.keep(cache, batch, w, 6000, 4, 9)
            assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])


def test_keep_with_budgets_of_their_own_and_wild_lengths(torch):
    """Budgets and lengths are the device's: below zero, above their bounds, zero."""
    from paper_2609_26219_amd import serving

    lens = (50, 50, 50, 50, 50, 0)
    cache, batch = _sequences(torch, lens, 1)
    w = np.random.default_rng(0).exponential(1.0, (6, 1, 50)).astype(np.float32)
    budgets = [7, 0, -3, 1000, 2 ** 31 - 1, 5]
    kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), 20, 2, 3, budgets=_dev(torch, budgets))
    want = os_.keep(w, lens, [min(b, 20) for b in budgets], 2, 3)
    assert kept_lens.tolist() == [7, 0, 0, 20, 20, 0]
    assert np.array_equal(kept.cpu().numpy(), _expect(want, 20, 1, 6))
    batch.keep[1].copy_(_dev(torch, [-1, 2 ** 31 - 1, 51, -2 ** 31, 1, 2]))
    kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), 20, 2, 3)
    want = os_.keep(w, [0, 50, 50, 0, 1, 2], [20] * 6, 2, 3)
    assert np.array_equal(kept.cpu().numpy(), _expect(want, 20, 1, 6)) and kept_lens.tolist() == [0, 20, 20, 0, 1, 2]
    kept, kept_lens = serving.keep(cache, batch, torch.from_numpy(w).cuda(), 0)
    assert kept.shape == (6, 1, 0) and not kept_lens.any()


def test_keep_strided_weights_and_given_outputs(torch):
    from paper_2609_26219_amd import serving

    lens = (90, 33)
    cache, batch = _sequences(torch, lens, 4)
    wide = torch.rand((2, 6, 128), device="cuda")
    w = wide[:, 1:5, 3:100]
    out = (torch.full((2, 4, 30), 9, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda"))
    got = serving.keep(cache, batch, w, 30, 1, 2, out=out)
    assert got is out
    want = os_.keep(w.cpu().numpy(), lens, [30, 30], 1, 2)
    assert np.array_equal(out[0].cpu().numpy(), _expect(want, 30, 4, 2))


EVICT = [
    # tag, dtype, H, D, P, lens, budget
    (K4V4, BF16, 2, 64, 16, (40, 3, 0, 17, 100), 20),
    (K8V4, HALF, 3, 128, 1, (95, 31), 31),
    (K8V8, BF16, 1, 256, 4, (130, 64), 100),
    (K4V4, HALF, 5, 96, 8, (90,), 1),
    (K4V4, HALF, 3, 48, 8, (90, 12), 40),
    (K8V4, BF16, 2, 16, 2, (64, 9), 30),
    (FP16, BF16, 8, 128, 32, (257, 64, 5), 64),
    (FP16, HALF, 3, 48, 8, (90, 91), 50),
    (FP16, BF16, 1, 512, 64, (200,), 77),
    (K4V4, BF16, 8, 512, 16, (33,), 16),
    (K4V4, BF16, 1, 64, 16, (5000, 2200), 2100),
    (FP16, HALF, 1, 64, 16, (1500,), 1300),
]


@pytest.mark.parametrize("tag,dtype,H,D,P,lens,budget", EVICT)
@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("moved", [False, True])
def test_evict(torch, tag, dtype, H, D, P, lens, budget, joint, moved):
    from paper_2609_26219_amd import serving

    rng = np.random.default_rng(D + budget)
    spare = sum(-(-min(n, budget) // P) for n in lens) + 3
    case = Case(41 + D + H, tag, dtype, H, 1, D, P, lens, (1,), layers=3, layer=1, spare_pages=spare)
    cache, batch = _cache(torch, case), _batch(torch, case)
    heads, S = 1 if joint else H, len(lens)
    w = rng.exponential(1.0, (S, heads, max(lens) + 3)).astype(np.float32)
    kept = os_.keep(w, lens, [budget] * S, 2, 5)
    free = [p for p in rng.permutation(case.pool) if p not in set(case.table[case.table >= 0])]
    to = case.table
    if moved:
        to = np.full((S, max(1, -(-budget // P))), -1, np.int32)
        for s, n in enumerate(lens):
            for i in range(-(-min(n, budget) // P)):
                to[s, i] = free.pop()
    want, want_w = os_.evict(case.cache, tag, P, kept, lens, case.table, to, w)
    dw = torch.from_numpy(w).cuda()
    serving.evict(cache, batch, _dev(torch, _expect(kept, budget, heads, S)), _dev(torch, [len(k[0]) for k in kept]), dw,
                  _dev(torch, to) if moved else None, layer=1)
    got, others = _state(torch, cache, case)
    for g, x in zip(got, want["kv"] if tag == FP16 else [want["codes"], want["scales"]]):
        assert np.array_equal(g.view(x.dtype), x)
    assert others and np.array_equal(dw.cpu().numpy(), want_w)


def test_evict_to_the_same_pages_is_in_place(torch):
    from paper_2609_26219_amd import serving

    case = Case(49, K4V4, BF16, 2, 1, 64, 16, (3000, 70), (1,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    w = np.random.default_rng(0).exponential(1.0, (2, 1, 3000)).astype(np.float32)
    kept = os_.keep(w, case.lens, [2500, 2500], 4, 4)
    want, _ = os_.evict(case.cache, K4V4, 16, kept, case.lens, case.table, case.table)
    serving.evict(cache, batch, _dev(torch, _expect(kept, 2500, 1, 2)), _dev(torch, [2500, 70]), page_table=batch.keep[2])
    for g, x in zip(_state(torch, cache, case)[0], [want["codes"], want["scales"]]):
        assert np.array_equal(g.view(x.dtype), x)


@pytest.mark.parametrize("paired", [False, True])
def test_evict_paired_pages(torch, paired):
    from paper_2609_26219_amd import serving

    case = Case(50, FP16, BF16, 4, 1, 64, 16, (200, 70), (1,), paired=paired)
    cache, batch = _cache(torch, case), _batch(torch, case)
    w = np.random.default_rng(0).exponential(1.0, (2, 4, 200)).astype(np.float32)
    kept = os_.keep(w, case.lens, [64, 64], 4, 4)
    want, _ = os_.evict(case.cache, FP16, 16, kept, case.lens, case.table, case.table)
    serving.evict(cache, batch, _dev(torch, _expect(kept, 64, 4, 2)), _dev(torch, [64, 64]))
    for g, x in zip(_state(torch, cache, case)[0], want["kv"]):
        assert np.array_equal(g.view(x.dtype), x)


@pytest.mark.parametrize("tag", [FP16, K4V4])
@pytest.mark.parametrize("moved", [False, True])
def test_evict_with_pages_that_are_not_there(torch, tag, moved):
    """Rows whose page is not there, before or after, are left out; indices outside the sequence too."""
    from paper_2609_26219_amd import serving

    case = Case(51, tag, BF16, 2, 1, 64, 4, (60, 45), (1,), holes=6, spare_pages=30)
    cache, batch = _cache(torch, case), _batch(torch, case)
    kept = np.full((2, 1, 25), -1, np.int32)
    kept[0, 0, :20] = np.sort(np.random.default_rng(1).permutation(60)[:20])
    kept[1, 0, :] = np.arange(20, 45)
    bad = kept.copy()
    bad[0, 0, 20:] = [60, 61, -5, 2 ** 31 - 1, -2 ** 31]
    rows = [[list(kept[0, 0, :20])], [list(kept[1, 0])]]
    to = case.table
    if moved:
        free = [p for p in range(case.pool) if p not in set(case.table[case.table >= 0])]
        to = np.array(free[:10], np.int32).reshape(2, 5)  # (fewer pages than rows)
        to[0, 1] = -1
        to[1, 2] = case.pool
    want, _ = os_.evict(case.cache, tag, 4, rows, case.lens, case.table, to)
    serving.evict(cache, batch, _dev(torch, bad), _dev(torch, [25, 2 ** 30]), page_table=_dev(torch, to) if moved else None)
    for g, x in zip(_state(torch, cache, case)[0], want["kv"] if tag == FP16 else [want["codes"], want["scales"]]):
        assert np.array_equal(g.view(x.dtype), x)


def test_evict_within_the_budget_changes_nothing(torch):
    from paper_2609_26219_amd import serving

    case = Case(52, K8V4, HALF, 2, 1, 64, 16, (30, 0, 1), (1,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    w = torch.rand((3, 2, 30), device="cuda")
    before = cache.codes.clone(), cache.scales.clone(), w.clone()
    kept, kept_lens = serving.keep(cache, batch, w, 40)
    serving.evict(cache, batch, kept, kept_lens, w)
    assert kept_lens.tolist() == [30, 0, 1]
    assert torch.equal(cache.codes, before[0]) and torch.equal(w, before[2])
    assert torch.equal(cache.scales.view(torch.int16), before[1].view(torch.int16))


@pytest.mark.parametrize("tag,dtype", [(K4V4, BF16), (FP16, HALF)])
@pytest.mark.parametrize("joint", [False, True])
def test_a_decode_loop_over_a_bounded_cache(torch, tag, dtype, joint):
    """Rotate and append, attend, weigh; every few steps keep and evict, the offsets following; replayed from two graphs
    (a step, an eviction), as lengths, offsets and rows change, against the same calls made eagerly on another cache, and
    the state of the oracle at each eviction."""
    from paper_2609_26219_amd import serving

    H, group, D, P, budget = 2, 4, 64, 16, 40
    lens = (55, 20, 41)
    heads = 1 if joint else H
    made = []
    for _ in range(2):
        case = Case(60, tag, dtype, H, group, D, P, lens, (1,), wide=4, spare_pages=20)
        free = iter([p for p in range(case.pool) if p not in set(case.table[case.table >= 0])])
        for s, n in enumerate(lens):
            for i in range(-(-n // P), min(case.table.shape[1], -(-(n + 12) // P))):
                case.table[s, i] = next(free)
        cache = _cache(torch, case)
        kv_lens, offset = _dev(torch, lens), _dev(torch, [0, 0, 0])
        top = case.table.shape[1] * P
        batch = serving.Batch(_dev(torch, [0, 1, 2, 3]), kv_lens, _dev(torch, case.table), 3, max_tokens=1, max_kv_len=top)
        q, k, v = (torch.empty((3, n, D), dtype=torch.float16 if dtype == HALF else torch.bfloat16, device="cuda")
                   for n in (H * group, H, H))
        w = torch.zeros((3, heads, top), device="cuda")
        out, turned = torch.empty_like(q), torch.empty_like(q)
        kept = (torch.empty((3, heads, budget), dtype=torch.int32, device="cuda"),
                torch.empty(3, dtype=torch.int32, device="cuda"))

        def step(cache=cache, batch=batch, kv_lens=kv_lens, offset=offset, q=q, k=k, v=v, w=w, out=out, turned=turned):
            kv_lens.add_(1)
            serving.append_rotated(cache, batch, q, k, v, out=turned, position_offset=offset)
            _, lse = serving.attention(cache, batch, turned, out=out, return_lse=True)
            serving.attention_weights(cache, batch, turned, lse, w, w, decay=0.9)

        def cut(cache=cache, batch=batch, kv_lens=kv_lens, offset=offset, w=w, kept=kept):
            serving.keep(cache, batch, w, budget, sinks=2, recent=8, out=kept)
            serving.evict(cache, batch, *kept, w)
            offset.add_(kv_lens).sub_(kept[1])
            kv_lens.copy_(kept[1])

        made.append((case, cache, batch, kv_lens, offset, (q, k, v), w, out, kept, step, cut))
    eager, captured = made
    case, cache = captured[:2]
    before = [t.clone() for t in ((cache.codes, cache.scales) if tag else (cache.k_cache, cache.v_cache))]
    for call in captured[9:]:  # (first calls outside the capture, undone)
        call()
    graphs = []
    for call in captured[9:]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for t, b in zip((cache.codes, cache.scales) if tag else (cache.k_cache, cache.v_cache), before):
        t.copy_(b)
    captured[3].copy_(eager[3])
    captured[4].zero_()
    captured[6].zero_()
    gen = torch.Generator(device="cuda").manual_seed(2)
    state = lambda m: [*_state(torch, m[1], m[0])[0], *(t.cpu().numpy() for t in (m[3], m[4], m[6])), _down(m[7])]  # noqa: E731
    total = np.array(lens)
    for i in range(24):
        for a, b in zip(eager[5], captured[5]):
            a.copy_(torch.randn(a.shape, generator=gen, device="cuda"))
            b.copy_(a)
        eager[9]()
        graphs[0].replay()
        total = total + 1
        if i % 5 == 4:
            at = state(eager)
            now = {"kv": at[:2]} if tag == FP16 else {"codes": at[0], "scales": at[1].view(np.uint16).reshape(
                case.cache["scales"].shape)}
            stay = os_.keep(at[-2], at[-4], [budget] * 3, 2, 8)
            want, want_w = os_.evict(now, tag, P, stay, at[-4], eager[0].table, eager[0].table, at[-2])
            eager[10]()
            graphs[1].replay()
            got = state(eager)
            for g, x in zip(got, want["kv"] if tag == FP16 else [want["codes"], want["scales"]]):
                assert np.array_equal(g.view(x.dtype).reshape(x.shape), x)
            assert np.array_equal(got[-2], want_w)
            assert (got[-4] <= budget).all()
        a, b = state(eager), state(captured)
        assert all(np.array_equal(x, y) for x, y in zip(a, b))
        assert (a[-4] + a[-3] == total).all()  # places and offset together count every token there was
        assert np.isfinite(a[-2]).all()


def test_refusals(torch):
    from paper_2609_26219_amd import serving

    case = Case(53, K4V4, BF16, 2, 1, 64, 16, (30, 9), (1,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    w = torch.rand((2, 2, 30), device="cuda")
    kept, kept_lens = serving.keep(cache, batch, w, 8)
    for args, kw in (((w[:1], 8), {}), ((w.double(), 8), {}), ((w, 8), dict(budgets=torch.zeros(3, dtype=torch.int32).cuda())),
                     ((w, 8), dict(out=(kept[:, :1].contiguous(), kept_lens))), ((w, 9), dict(out=(kept, kept_lens))),
                     ((w, 8), dict(out=(kept.long(), kept_lens))), ((w, -1), {})):
        with pytest.raises(ValueError):
            serving.keep(cache, batch, *args, **kw)
    for args, kw in (((w[..., :29], 8), {}), ((w, 8), dict(sinks=-1)), ((w, 8), dict(recent=-1)), ((w.cpu(), 8), {})):
        with pytest.raises(pb.PkvError):
            serving.keep(cache, batch, *args, **kw)
    with pytest.raises(ValueError):
        serving.evict(cache, batch, kept.float(), kept_lens)
    with pytest.raises(ValueError):
        serving.evict(cache, batch, kept, kept_lens[:1])
    with pytest.raises(ValueError):
        serving.evict(cache, batch, kept, kept_lens, page_table=torch.zeros((1, 4), dtype=torch.int32, device="cuda"))
    for kw in (dict(layer=1), dict(weights=w[:, :1]), dict(weights=w[..., :29])):
        with pytest.raises(pb.PkvError):
            serving.evict(cache, batch, kept, kept_lens, **kw)
    with pytest.raises(pb.PkvError):
        serving.evict(cache, batch, kept.cpu(), kept_lens)


@pytest.mark.parametrize("tag", [FP16, K8V8])
def test_offsets_past_32_bits(torch, tag):
    """A cache whose used pages lie past 4 GiB from its start: rows turned and appended, weighed and moved there are those of a
    small cache."""
    from paper_2609_26219_amd import serving

    H, D, P, n = 8, 256, 64, 300
    need, pool = 5, 20000 if tag == FP16 else 9000
    made = []
    for pages in (need + 5, pool):
        kw = dict(num_kv_heads=H, head_dim=D, page_size=P, dtype=torch.bfloat16, tag=tag)
        if tag == FP16:
            cache = serving.PagedCache(k_cache=torch.zeros((pages, P, H, D), dtype=torch.bfloat16, device="cuda"),
                                       v_cache=torch.zeros((pages, P, H, D), dtype=torch.bfloat16, device="cuda"), **kw)
        else:
            cache = serving.PagedCache(pool_pages=pages, **kw)
        table = torch.arange(pages - need, pages, dtype=torch.int32, device="cuda").flip(0).contiguous()[None]
        other = torch.arange(pages - need - 5, pages - need, dtype=torch.int32, device="cuda")[None].contiguous()
        made.append((cache, table, other))
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((n, h, D), generator=gen, device="cuda").bfloat16() for h in (2 * H, H, H))
    got = []
    for cache, table, other in made:
        batch = serving.Batch(_dev(torch, [0, n]), _dev(torch, [n]), table, n, max_kv_len=n)
        turned = serving.append_rotated(cache, batch, q, k, v)
        last = serving.Batch(_dev(torch, [0, 1]), _dev(torch, [n]), table, 1, max_tokens=1, max_kv_len=n)
        w = torch.zeros((1, H, n), device="cuda")
        for b, rows in ((batch, turned), (last, turned[-1:])):
            _, lse = serving.attention(cache, b, rows, return_lse=True)
            serving.attention_weights(cache, b, rows, lse, w, w)
        kept = serving.keep(cache, last, w, 100, 2, 9)
        serving.evict(cache, last, *kept, page_table=other)
        moved = serving.read(cache, serving.Batch(_dev(torch, [0, 100]), _dev(torch, [100]), other, 100))
        weights = w.clone()
        serving.evict(cache, last, *kept, w)
        here = serving.read(cache, serving.Batch(_dev(torch, [0, 100]), _dev(torch, [100]), table, 100))
        got.append((turned, weights, *kept, w, *moved, *here))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    small = got[0]
    assert torch.equal(small[5], small[7]) and torch.equal(small[6], small[8]) and small[5].float().abs().sum() > 0


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("moved", [False, True])
def test_weights_at_indices_outside_are_left_out(torch, heads, moved):
    """As the rows there: the weight at such a place stays what it was.  A row whose page is not there moves its weight all
    the same."""
    from paper_2609_26219_amd import serving

    case = Case(54, K4V4, BF16, 2, 1, 64, 4, (20, 9000), (1,), spare_pages=8)
    case.table[0, 7 // 4] = -1
    cache, batch = _cache(torch, case), _batch(torch, case)
    w = np.random.default_rng(2).exponential(1.0, (2, heads, 9000)).astype(np.float32)
    kept = np.full((2, heads, 8500), -1, np.int32)
    kept[0, :, :6] = [3, 20, 7, -5, 9, 2 ** 31 - 1]
    kept[1] = np.arange(500, 9000)
    kept[1, :, [17, 8192, 8499]] = [[9000], [-1], [-2 ** 31]]
    want = w.copy()
    want[0, :, [0, 2, 4]] = w[0, :, [3, 7, 9]]
    want[0, :, 6:20] = 0.0
    stay = np.isin(np.arange(8500), [17, 8192, 8499])
    want[1, :, :8500] = np.where(stay, w[1, :, :8500], w[1, :, 500:])
    want[1, :, 8500:] = 0.0
    free = [p for p in range(case.pool) if p not in set(case.table[case.table >= 0])]
    to = _dev(torch, np.array(free[:2], np.int32).reshape(2, 1)) if moved else None
    dw = torch.from_numpy(w).cuda()
    serving.evict(cache, batch, _dev(torch, kept), _dev(torch, [6, 8500]), dw, to)
    assert np.array_equal(dw.cpu().numpy(), want)


def test_codes_past_4_gib(torch):
    """Codes whose pages lie past 4 GiB from the cache's start: rows turned and appended, weighed and moved there (in place
    and to other pages) are those of a small cache."""
    from paper_2609_26219_amd import serving

    H, D, P, n, need, pool = 8, 256, 64, 300, 5, 20000
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((n, h, D), generator=gen, device="cuda").bfloat16() for h in (2 * H, H, H))
    got = []
    for pages in (2 * need, pool):
        cache = serving.PagedCache(H, D, P, torch.bfloat16, K8V8, pool_pages=pages)
        used = pages - 2 * need
        assert pages != pool or used * (cache.codes.numel() // pages) > 2 ** 32
        other = torch.arange(used, used + need, dtype=torch.int32, device="cuda")[None].contiguous()
        table = (other + need).flip(1).contiguous()
        batch = serving.Batch(_dev(torch, [0, n]), _dev(torch, [n]), table, n, max_kv_len=n)
        last = serving.Batch(_dev(torch, [0, 1]), _dev(torch, [n]), table, 1, max_tokens=1, max_kv_len=n)
        turned = serving.append_rotated(cache, batch, q, k, v)
        w = torch.zeros((1, H, n), device="cuda")
        for b, rows in ((batch, turned), (last, turned[-1:])):
            _, lse = serving.attention(cache, b, rows, return_lse=True)
            serving.attention_weights(cache, b, rows, lse, w, w)
        kept = serving.keep(cache, last, w, 100, 2, 9)
        serving.evict(cache, last, *kept, page_table=other)
        weights = w.clone()
        serving.evict(cache, last, *kept, w)
        got.append((turned, weights, *kept, w, cache.codes[:, used:].clone(), cache.scales[:, used:].view(torch.int16).clone()))
        assert not cache.codes[:, :used].any()
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][5].any()
