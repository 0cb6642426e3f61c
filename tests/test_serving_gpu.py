"""The serving calls on the GPU against the fp64 oracle: rows written into a paged cache (codes and scales bit for
bit), read back, and attention over it at the sizes, masks and layouts where such kernels go wrong."""
import numpy as np
import pytest

from paper_2609_26219_amd import binding as pb
from paper_2609_26219_amd import workloads as wl
from serving_cases import Case, check_attention, check_read

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


def _dtype(torch, case):
    return torch.bfloat16 if case.dtype else torch.float16


def _up(torch, bits, case):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(_dtype(torch, case))


def _down(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _cache(torch, case):
    """The case's cache on the device, other layers filled with 0x5A."""
    from paper_2609_26219_amd import serving

    def layered(a):
        t = torch.full((case.layers, *a.shape), 0x5A, dtype=torch.uint8 if a.dtype == np.uint8 else torch.int16,
                       device="cuda")
        t[case.layer] = torch.from_numpy(a if a.dtype == np.uint8 else a.view(np.int16)).cuda()
        return t

    kw = dict(num_kv_heads=case.H, head_dim=case.D, page_size=case.P, dtype=_dtype(torch, case), tag=case.tag)
    if case.tag == FP16:
        k, v = (layered(a) for a in case.cache["kv"])
        if case.paired:
            both = torch.stack([k, v], 2)
            k, v = both[:, :, 0], both[:, :, 1]
        return serving.PagedCache(k_cache=k, v_cache=v, **kw)
    return serving.PagedCache(codes=layered(case.cache["codes"]),
                              scales=layered(case.cache["scales"]).view(torch.float16), **kw)


def _batch(torch, case, bounds=True):
    from paper_2609_26219_amd import serving
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    return serving.Batch(dev(case.start), dev(case.lens), dev(case.table), case.tokens, dev(case.positions),
                         case.most_new if bounds else 0, case.most_kv if bounds else 0)


def _state(torch, cache, case):
    """The layer of the case as host arrays, and whether every other layer is untouched."""
    if case.tag == FP16:
        ts = [cache.k_cache, cache.v_cache]
    else:
        ts = [cache.codes, cache.scales]
    host = [t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.uint8).cpu().numpy() for t in ts]
    others = all((np.delete(h, case.layer, 0) == 0x5A).all() for h in host)
    return [h[case.layer] for h in host], others


APPEND = [
    # tag, dtype, H, D, P, lens, new
    (K4V4, BF16, 2, 64, 16, (40, 3, 0, 17), (5, 3, 1, 17)),
    (K8V4, HALF, 3, 128, 1, (9,), (9,)),
    (K8V8, BF16, 1, 256, 4, (33, 1), (33, 1)),
    (K4V4, HALF, 5, 96, 8, (21, 8), (7,)),
    (K8V4, BF16, 2, 16, 2, (13,), (13,)),
    (K4V4, HALF, 8, 512, 32, (70,), (70,)),
    (FP16, BF16, 2, 128, 16, (31, 2), (9, 2)),
    (FP16, HALF, 3, 48, 1, (5,), (5,)),
    (K4V4, BF16, 8, 128, 64, tuple(range(1, 41)), (1,)),
]


@pytest.mark.parametrize("tag,dtype,H,D,P,lens,new", APPEND)
@pytest.mark.parametrize("scattered", [False, True])
def test_append_is_the_definition_bit_for_bit(torch, tag, dtype, H, D, P, lens, new, scattered):
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    case = Case(11 + D, tag, dtype, H, 1, D, P, lens, new, scattered=scattered, holes=1, layers=3, layer=1)
    cache, batch = _cache(torch, case), _batch(torch, case)
    serving.append(cache, batch, _up(torch, case.k, case), _up(torch, case.v, case), layer=1)
    want = case.copy_of_cache()
    os_.append(want, tag, P, case.where(), case.k, case.v, dtype)
    got, others = _state(torch, cache, case)
    names = want["kv"] if tag == FP16 else [want["codes"], want["scales"]]
    for g, w in zip(got, names):
        assert np.array_equal(g.view(w.dtype), w)
    assert others


def _special_rows(dtype):
    """Rows whose range or codes sit where roundings go wrong: constants, signed zeros, extremes, ties, subnormals."""
    rng = np.random.default_rng(5)
    rows = [np.zeros(64), -np.zeros(64), np.full(64, 1.5), np.full(64, -2.0 ** -14), np.full(64, 65504.0 if not dtype else 65280.0)]
    ramp = np.arange(64) / 4.0
    rows += [ramp, -ramp, ramp * 2.0 ** -20, np.where(np.arange(64) % 2, 65280.0, -65280.0)]
    rows += [np.concatenate([[-1.0, 6.5], rng.integers(0, 16, 62) * 0.5 - 0.75])]  # quotients at half-integers
    rows += [np.concatenate([[0.0, 15.0], rng.integers(0, 30, 62) * 0.5])]
    rows += [np.concatenate([[0.0, 255.0], rng.integers(0, 510, 62) * 0.5])]
    rows += [rng.standard_normal(64) * 10.0 ** e for e in (-7, -5, -3, 2, 4)]
    rows += [np.where(np.arange(64) % 3 == 0, -0.0, 2.0 ** -24)]
    return np.clip(np.stack(rows), -65280, 65504 if not dtype else 65280)


@pytest.mark.parametrize("tag", [K8V8, K4V4])
@pytest.mark.parametrize("dtype", [HALF, BF16])
def test_append_rows_at_the_edges_of_the_rule(torch, tag, dtype):
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    rows = _special_rows(dtype)
    n = len(rows)
    case = Case(3, tag, dtype, 1, 1, 64, 16, (n,), (n,))
    case.k, case.v = case.bits(rows)[:, None], case.bits(rows[::-1])[:, None]
    cache, batch = _cache(torch, case), _batch(torch, case)
    serving.append(cache, batch, _up(torch, case.k, case), _up(torch, case.v, case))
    want = case.copy_of_cache()
    os_.append(want, tag, 16, case.where(), case.k, case.v, dtype)
    (codes, scales), _ = _state(torch, cache, case)
    assert np.array_equal(scales.view(np.uint16), want["scales"])
    assert np.array_equal(codes, want["codes"])


@pytest.mark.parametrize("tag,dtype,H,D,P,lens,new", APPEND)
def test_read_back(torch, tag, dtype, H, D, P, lens, new):
    from paper_2609_26219_amd import serving

    case = Case(21 + D, tag, dtype, H, 1, D, P, lens, new, holes=1, layers=2, layer=1)
    cache, batch = _cache(torch, case), _batch(torch, case)
    k, v = serving.read(cache, batch, layer=1)
    for which, t in enumerate((k, v)):
        check_read(case, _down(t), which)


def test_rows_at_strides(torch):
    """k and v as slices of one fused buffer, in and out; bytes between the rows stay."""
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    case = Case(77, K8V4, BF16, 2, 1, 64, 16, (40, 9), (11, 9))
    cache, batch = _cache(torch, case), _batch(torch, case)
    fused = torch.full((case.tokens, 7, 80), -3.0, dtype=torch.bfloat16, device="cuda")
    k, v = fused[:, 1:3, :64], fused[:, 4:6, :64]
    k.copy_(_up(torch, case.k, case))
    v.copy_(_up(torch, case.v, case))
    serving.append(cache, batch, k, v)
    want = case.copy_of_cache()
    os_.append(want, K8V4, 16, case.where(), case.k, case.v, BF16)
    (codes, scales), _ = _state(torch, cache, case)
    assert np.array_equal(codes, want["codes"]) and np.array_equal(scales.view(np.uint16), want["scales"])
    case.cache = want
    fused.fill_(-3.0)
    serving.read(cache, batch, out=(k, v))
    check_read(case, _down(k), 0)
    check_read(case, _down(v), 1)
    mask = torch.ones_like(fused, dtype=torch.bool)
    mask[:, 1:3, :64] = False
    mask[:, 4:6, :64] = False
    assert (fused[mask] == -3.0).all()


def test_rows_of_no_sequence_are_left_alone(torch):
    from paper_2609_26219_amd import serving

    case = Case(78, K4V4, HALF, 2, 2, 64, 16, (20, 30), (4, 6))
    cache, batch = _cache(torch, case), _batch(torch, case)
    batch.keep[0].copy_(torch.tensor([2, 5, 8], dtype=torch.int32))  # rows 0, 1, 8 and 9 belong to nobody
    before = [t.clone() for t in (cache.codes, cache.scales)]
    k = torch.full((10, 2, 64), 7.0, dtype=torch.float16, device="cuda")
    v = k.clone()
    serving.read(cache, batch, out=(k, v))
    out = torch.full((10, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    serving.attention(cache, batch, _up(torch, case.q, case), out=out)
    for t in (k, v, out):
        assert (t[[0, 1, 8, 9]] == 7.0).all() and (t[2:8] != 7.0).any()
    case.start = np.array([2, 5, 8], np.int32)
    check_read(case, _down(k), 0)
    serving.append(cache, batch, k, v)  # nothing but the six rows
    changed = (cache.scales.view(torch.int16) != before[1].view(torch.int16)).any(-1).any(3).any(2)[0]
    assert {tuple(at) for at in changed.nonzero().tolist()} == {(p, slot) for _, _, p, slot in case.where() if p >= 0}


ATTEND = [
    # tag, dtype, H, group, D, P, lens, new, scattered, window, sinks
    (K4V4, HALF, 2, 4, 64, 16, (1,), (1,), False, 0, 0),
    (K4V4, BF16, 2, 4, 128, 16, (77, 0, 5, 32, 33, 31), (1,), False, 0, 0),
    (K4V4, BF16, 1, 1, 256, 32, (65, 130), (2, 3), False, 0, 0),
    (K8V4, HALF, 2, 3, 128, 16, (50, 200), (17, 40), False, 0, 0),
    (K8V8, BF16, 1, 5, 64, 64, (100,), (100,), False, 0, 0),
    (K4V4, HALF, 2, 2, 128, 1, (45, 3), (3, 3), False, 0, 0),
    (K8V4, BF16, 1, 8, 64, 2, (39,), (5,), False, 9, 2),
    (K4V4, HALF, 1, 2, 256, 8, (70, 12), (12,), False, 16, 4),
    (K4V4, BF16, 2, 4, 128, 16, (300, 40), (1,), False, 64, 4),
    (K8V8, HALF, 2, 1, 128, 16, (150,), (33,), True, 0, 0),
    (FP16, BF16, 2, 4, 128, 16, (77, 0, 5, 32), (1,), False, 0, 0),
    (FP16, HALF, 1, 4, 64, 16, (300, 17), (40, 17), False, 50, 3),
    (FP16, BF16, 2, 2, 256, 4, (40, 90), (8, 1), False, 0, 0),
    (FP16, BF16, 1, 16, 128, 32, (200,), (20,), True, 30, 40),
    (FP16, HALF, 2, 1, 128, 1, (33,), (33,), False, 5, 0),
    (FP16, BF16, 1, 1, 64, 64, (513,), (1,), False, 1, 0),
    (FP16, HALF, 1, 2, 128, 16, (290,), (290,), False, 0, 0),
    (K4V4, BF16, 1, 4, 128, 16, (1500, 700), (1,), False, 0, 0),
    (FP16, BF16, 1, 4, 128, 16, (1500, 10), (1,), False, 200, 1000),
    (K8V4, BF16, 1, 2, 128, 16, (400,), (130,), True, 40, 5),
    (FP16, HALF, 1, 3, 256, 16, (70, 200), (23, 31), False, 0, 0),
    (FP16, BF16, 1, 1, 256, 2, (90,), (60,), True, 11, 3),
    (K4V4, BF16, 2, 8, 64, 16, (33, 170), (4,), False, 0, 0),
    (K8V8, HALF, 1, 8, 128, 16, (400, 9, 31), (4, 2, 4), False, 100, 7),
    (FP16, BF16, 2, 8, 128, 8, (33, 170), (4,), False, 0, 0),
    (K8V4, HALF, 1, 1, 64, 1, (260, 5), (140, 5), False, 128, 1),
    (K4V4, BF16, 1, 4, 128, 16, (700,), (65,), True, 33, 70),
]


@pytest.mark.parametrize("tag,dtype,H,group,D,P,lens,new,scattered,window,sinks", ATTEND)
@pytest.mark.parametrize("holes", [0, 2])
def test_attention(torch, tag, dtype, H, group, D, P, lens, new, scattered, window, sinks, holes):
    from paper_2609_26219_amd import serving

    case = Case(31 + D + window, tag, dtype, H, group, D, P, lens, new, scattered=scattered, holes=holes, layers=2,
                layer=1, paired=tag == FP16 and P == 16, wide=holes)
    cache = _cache(torch, case)
    for bounds in (True, False):
        out, lse = serving.attention(cache, _batch(torch, case, bounds), _up(torch, case.q, case), window=window,
                                     sinks=sinks, layer=1, return_lse=True)
        check_attention(case, _down(out), lse.cpu().numpy(), window, sinks)


@pytest.mark.parametrize("tag,values", [(K4V4, 1e-3), (K4V4, 300.0), (K8V4, 1e-5), (FP16, 1e-4)])
@pytest.mark.parametrize("dtype", [HALF, BF16])
def test_attention_of_small_and_large_values(torch, tag, values, dtype):
    """Scales near binary16's ends, scores far apart or all alike."""
    from paper_2609_26219_amd import serving

    case = Case(41, tag, dtype, 1, 4, 128, 16, (90, 400), (3, 1), scale_of_values=values)
    scale = 0.1 / values ** 2 if values < 1 else 1e-5
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), scale=scale,
                                 return_lse=True)
    check_attention(case, _down(out), lse.cpu().numpy(), scale=scale)


def test_attention_at_positions_past_the_cache(torch):
    """Positions beyond kv_lens: only what is cached and in the window counts, so some rows keep their sinks alone or
    see nothing; negative positions see nothing."""
    from paper_2609_26219_amd import serving

    case = Case(43, FP16, BF16, 1, 2, 64, 16, (40, 70), (5, 4))
    case.positions = np.array([39, 100, 45, -1, 0, 500, 69, -2 ** 31, 2 ** 31 - 1], np.int32)
    for window, sinks in ((0, 0), (20, 3), (20, 0), (7, 100)):
        out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), window=window,
                                     sinks=sinks, return_lse=True)
        check_attention(case, _down(out), lse.cpu().numpy(), window, sinks)


def test_attention_at_strides_and_into_out(torch):
    from paper_2609_26219_amd import serving

    case = Case(47, K4V4, BF16, 2, 2, 128, 16, (60, 9), (2, 9))
    cache, batch = _cache(torch, case), _batch(torch, case)
    fused = torch.full((case.tokens, 9, 136), 2.0, dtype=torch.bfloat16, device="cuda")
    q, out = fused[:, :4, :128], fused[:, 5:, :128]
    q.copy_(_up(torch, case.q, case))
    got, lse = serving.attention(cache, batch, q, out=out, return_lse=True)
    assert got is out
    check_attention(case, _down(out), lse.cpu().numpy())
    assert (fused[:, 4] == 2.0).all() and (fused[:, :, 128:] == 2.0).all()


def test_infinities_and_nans_in_unseen_places_do_not_matter(torch):
    """Values that no row sees, in pages that rows do see: past the end, before the window, behind the sinks."""
    from paper_2609_26219_amd import serving

    case = Case(53, FP16, HALF, 1, 4, 64, 16, (100,), (1,))
    clean = case.copy_of_cache()
    for t in list(range(5, 60)):
        p, s = case.table[0, t // 16], t % 16
        for a in case.cache["kv"]:
            a[p, s] = [0x7E00, 0x7C00, 0xFC00][t % 3]
    dirty, case.cache = case.cache, clean
    window, sinks = 40, 5
    batch = _batch(torch, case)
    case.cache = dirty
    out, lse = serving.attention(_cache(torch, case), batch, _up(torch, case.q, case), window=window, sinks=sinks,
                                 return_lse=True)
    case.cache = clean
    check_attention(case, _down(out), lse.cpu().numpy(), window, sinks)


def test_cache_past_four_gibibytes(torch):
    """Pages whose byte offsets pass 32 bits, quantised and 16-bit."""
    from paper_2609_26219_amd import serving

    for tag in (K4V4, FP16):
        case = Case(59, tag, BF16, 8, 2, 128, 16, (50, 20), (1,))
        far = 700_000 if tag != FP16 else 300_000  # 16 KiB of codes, 64 KiB of K and V a page
        kw = dict(num_kv_heads=8, head_dim=128, page_size=16, dtype=torch.bfloat16, tag=tag)
        up = lambda a: torch.from_numpy(a if a.dtype == np.uint8 else a.view(np.int16)).cuda()  # noqa: E731
        if tag == FP16:
            kv = torch.empty((far + case.pool, 2, 16, 8, 128), dtype=torch.bfloat16, device="cuda")
            for which in range(2):
                kv[far:, which] = up(case.cache["kv"][which]).view(torch.bfloat16)
            cache = serving.PagedCache(k_cache=kv[:, 0], v_cache=kv[:, 1], **kw)
        else:
            codes = torch.empty((far + case.pool, 8, 16 * 128), dtype=torch.uint8, device="cuda")
            scales = torch.empty((far + case.pool, 8, 2, 16, 2), dtype=torch.float16, device="cuda")
            codes[far:], scales[far:] = up(case.cache["codes"]), up(case.cache["scales"]).view(torch.float16)
            cache = serving.PagedCache(codes=codes, scales=scales, **kw)
        batch = _batch(torch, case)
        table = batch.keep[2]
        table.copy_(torch.where(table >= 0, table + far, table))
        out, lse = serving.attention(cache, batch, _up(torch, case.q, case), return_lse=True)
        check_attention(case, _down(out), lse.cpu().numpy())
        k, v = serving.read(cache, batch)
        check_read(case, _down(k), 0)
        check_read(case, _down(v), 1)
        serving.append(cache, batch, k, v)
        again, _ = serving.read(cache, batch)
        assert (again.float() - k.float()).abs().max() <= 0.6  # one more quantisation: within a 4-bit step
        del cache
        torch.cuda.empty_cache()


def test_other_stream_and_graph(torch):
    """On a side stream, and replayed from a graph while lengths, tables and rows change in place."""
    from paper_2609_26219_amd import serving

    case = Case(61, K4V4, BF16, 2, 4, 128, 16, (900, 300), (1,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    q, k, v = (_up(torch, b, case) for b in (case.q, case.k, case.v))

    def step(out):
        serving.append(cache, batch, k, v)
        return serving.attention(cache, batch, q, out=out)

    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    side.synchronize()
    from oracle import serving as os_
    os_.append(case.cache, K4V4, 16, case.where(), case.k, case.v, BF16)
    exact = case.attend()
    check = lambda: check_attention(case, _down(out), exact[1].astype(np.float32))  # noqa: E731
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(out)
    for lens in ((900, 300), (37, 299), (512, 1)):
        out.zero_()
        case.lens = np.array(lens, np.int32)
        batch.keep[1].copy_(torch.tensor(lens, dtype=torch.int32))
        rng = np.random.default_rng(lens[0])
        case.q = case.bits(rng.standard_normal(case.q.shape))
        case.k = case.bits(rng.standard_normal(case.k.shape))
        q.copy_(_up(torch, case.q, case))
        k.copy_(_up(torch, case.k, case))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        os_.append(case.cache, K4V4, 16, case.where(), case.k, case.v, BF16)
        exact = case.attend()
        check()


def test_same_inputs_same_bits(torch):
    from paper_2609_26219_amd import serving

    case = Case(67, K8V4, BF16, 2, 4, 128, 16, (1400, 90), (1,))
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    first, lse = serving.attention(cache, batch, q, return_lse=True)
    for _ in range(3):
        again, lse2 = serving.attention(cache, batch, q, return_lse=True)
        assert torch.equal(first, again) and torch.equal(lse, lse2)


def test_refusals_on_the_device(torch):
    """Host memory, another tag's buffers and short buffers are refused before anything is enqueued."""
    from paper_2609_26219_amd import serving

    case = Case(71, K4V4, BF16, 2, 2, 64, 16, (20,), (2,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    q = _up(torch, case.q, case)
    with pytest.raises(pb.PkvError) as e:
        serving.attention(cache, batch, q, out=torch.empty(q.shape, dtype=q.dtype))
    assert e.value.status == pb.PKV_ERR_INVALID_ARGUMENT
    host = torch.from_numpy(case.lens)
    batch.struct.kv_lens = host.data_ptr()
    with pytest.raises(pb.PkvError):
        serving.attention(cache, batch, q)
    with pytest.raises(ValueError):
        serving.attention(cache, batch, q.float())
    with pytest.raises(ValueError):
        serving.append(cache, batch, q, q)


def _lengths(n, low, high, also=()):
    rng = np.random.default_rng(n)
    return (*also, *(int(x) for x in rng.integers(low, high, n)))


SPREAD = [
    # tag, dtype, H, group, D, P, lens, new, scattered, window, sinks: more sequences than a wave has lanes, cut into pieces and whole
    (K4V4, BF16, 2, 4, 64, 16, _lengths(150, 0, 60, (900,)), (1,), False, 0, 0),
    (FP16, HALF, 1, 2, 64, 16, _lengths(129, 0, 40, (700, 0, 0, 501)), (1, 2, 1), False, 0, 0),
    (K8V4, HALF, 1, 1, 64, 8, _lengths(70, 1, 300), (1,), False, 0, 0),
    (K4V4, BF16, 2, 7, 128, 16, (3000, 11, 2047), (3, 1, 4), False, 0, 0),
    (K8V8, BF16, 3, 5, 128, 16, (1700,), (1,), False, 0, 0),
    (FP16, BF16, 2, 3, 128, 32, (3000, 400), (2,), False, 1500, 40),
    (K4V4, HALF, 1, 8, 256, 16, (1200, 33), (2, 1), False, 0, 0),
    (FP16, HALF, 1, 2, 128, 16, (2000,), (4,), True, 700, 9),
    # many rows whose tokens are split, between two to 16 workgroups and more
    (FP16, BF16, 1, 1, 128, 64, (20001,), (40,), False, 0, 0),
    (K4V4, HALF, 1, 2, 128, 32, (2500, 300), (33, 20), False, 0, 0),
    (K8V4, BF16, 2, 5, 64, 16, (5003,), (9,), False, 0, 0),
    (FP16, HALF, 1, 2, 256, 16, (1203, 0), (30,), False, 0, 0),
    (K8V8, HALF, 1, 4, 256, 16, (9001,), (10,), True, 0, 0),
]


@pytest.mark.parametrize("tag,dtype,H,group,D,P,lens,new,scattered,window,sinks", SPREAD)
def test_attention_spread_over_the_gpu(torch, tag, dtype, H, group, D, P, lens, new, scattered, window, sinks):
    test_attention(torch, tag, dtype, H, group, D, P, lens, new, scattered, window, sinks, 1)


@pytest.mark.parametrize("tag", [K4V4, FP16])
def test_append_and_read_of_more_sequences_than_are_searched_in_lds(torch, tag):
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    case = Case(61, tag, BF16, 1, 1, 64, 4, _lengths(1100, 0, 6), (1, 2, 1))
    cache, batch = _cache(torch, case), _batch(torch, case)
    serving.append(cache, batch, _up(torch, case.k, case), _up(torch, case.v, case))
    want = case.copy_of_cache()
    os_.append(want, tag, 4, case.where(), case.k, case.v, BF16)
    got, _ = _state(torch, cache, case)
    for g, w in zip(got, want["kv"] if tag == FP16 else [want["codes"], want["scales"]]):
        assert np.array_equal(g.view(w.dtype), w)
    case.cache = want
    for which, t in enumerate(serving.read(cache, batch)):
        check_read(case, _down(t), which)


@pytest.mark.parametrize("tag,group,new", [(FP16, 4, 2), (K4V4, 2, 5), (K8V4, 8, 3)])
def test_windows_at_scattered_positions_of_many_sequences(torch, tag, group, new):
    """A window and positions: only the tokens between the rows' windows (and the sinks) are looked at, in pieces."""
    test_attention(torch, tag, BF16, 2, group, 64, 16, _lengths(70, 0, 90, (1800, 1, 0, 950)), (new, 1, new), True, 60, 5, 1)


@pytest.mark.parametrize("tag", [K8V8, K8V4, K4V4])
@pytest.mark.parametrize("new", [(1,), (130,)])
def test_binary16_results_over_codes_carry_the_results_rounding_alone(torch, tag, new):
    """Probabilities go in as two binary16 numbers, so what is left of their rounding is 2^-22 of each (2^-21 with the
    second's own underflow at 2^-38 of the largest, which check_attention's bound has as 2^-24 a token): its bound with
    that in the place of 2^-11.  Every row has an outlier 8 times its other channels."""
    from oracle.restore import output_values
    from paper_2609_26219_amd import serving

    case = Case(83, tag, HALF, 2, 4, 128, 16, (300, 777, 130), new)
    out, _ = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
    exact, _, mass, whole, reach = case.attend()
    have = output_values(_down(out), HALF)
    delta = 2.0 ** -23 * (case.D / 8 + 16) * reach
    tol = 2.0 ** -11 * np.abs(exact) * (1 + 2.0 ** -11) + (2.0 ** -21 + 2.0 ** -24 * case.most_kv) * mass + \
        (4 * delta + 2.0 ** -18)[:, :, None] * whole + 2.0 ** -25
    assert (np.abs(have - exact) <= tol).all(), float((np.abs(have - exact) / tol).max())


PAST = [
    # tag, group, lens, rows, bound: the forms of few rows, whole and in pieces, and of many rows, whole, split and split often
    (K4V4, 4, (300, 40), (5, 3), 2),
    (K4V4, 4, (3000, 40), (5, 3), 2),
    (FP16, 1, (200, 300), (90, 50), 45),
    (FP16, 1, (5000, 300), (60, 45), 45),
    (FP16, 1, (20001,), (60,), 45),
    (K8V4, 4, (5000, 300, 7), (45, 30, 7), 30),
]


@pytest.mark.parametrize("tag,group,lens,rows,bound", PAST)
def test_rows_past_the_bound_are_left_alone(torch, tag, group, lens, rows, bound):
    """Sequences with more rows than max_tokens says (a replayed graph's, say): the first of each are attended, the others
    keep what their places held."""
    from paper_2609_26219_amd import serving

    case = Case(91, tag, BF16, 1, group, 128, 16, lens, rows)
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    batch.struct.max_tokens = bound
    past = np.concatenate([np.arange(n) >= bound for n in rows])
    out = torch.full((case.tokens, group, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    _, lse = serving.attention(cache, batch, q, out=out, return_lse=True)
    assert past.any() and (out[torch.from_numpy(past).cuda()] == 7.0).all()
    # the rows within the bound, the others taken from a call that has them all
    whole, whole_lse = serving.attention(cache, _batch(torch, case), q, return_lse=True)
    out[torch.from_numpy(past).cuda()] = whole[torch.from_numpy(past).cuda()]
    lse[torch.from_numpy(past).cuda()] = whole_lse[torch.from_numpy(past).cuda()]
    check_attention(case, _down(out), lse.cpu().numpy())


@pytest.mark.parametrize("tag", [K4V4, FP16])
def test_starts_past_the_rows_of_the_call_are_their_number(torch, tag):
    """A last start beyond num_tokens counts as num_tokens for all three calls: the rows that are there are the last ones
    of their sequence, where they are written, read and attended from."""
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    case = Case(92, tag, BF16, 1, 2, 64, 16, (20, 30), (4, 6))
    cache, batch = _cache(torch, case), _batch(torch, case)
    batch.keep[0].copy_(torch.tensor([0, 4, 13], dtype=torch.int32))
    serving.append(cache, batch, _up(torch, case.k, case), _up(torch, case.v, case))
    want = case.copy_of_cache()
    os_.append(want, tag, 16, case.where(), case.k, case.v, BF16)
    got, _ = _state(torch, cache, case)
    for g, w in zip(got, want["kv"] if tag == FP16 else [want["codes"], want["scales"]]):
        assert np.array_equal(g.view(w.dtype), w)
    case.cache = want
    for which, t in enumerate(serving.read(cache, batch)):
        check_read(case, _down(t), which)
    out, lse = serving.attention(cache, batch, _up(torch, case.q, case), return_lse=True)
    check_attention(case, _down(out), lse.cpu().numpy())


def _check_fine(case, out, lse):
    """check_attention, and over codes with binary16 results its bound with 2^-21 in the place of 2^-11 (see
    test_binary16_results_over_codes_carry_the_results_rounding_alone)."""
    from oracle.restore import output_values

    check_attention(case, _down(out), lse.cpu().numpy())
    if case.dtype == HALF:
        exact, _, mass, whole, reach = case.attend()
        delta = 2.0 ** -23 * (case.D / 8 + 16) * reach
        tol = 2.0 ** -11 * np.abs(exact) * (1 + 2.0 ** -11) + (2.0 ** -21 + 2.0 ** -24 * case.most_kv) * mass + \
            (4 * delta + 2.0 ** -18)[:, :, None] * whole + 2.0 ** -25
        off = np.abs(output_values(_down(out), HALF) - exact)
        assert (off <= tol).all(), float((off / tol).max())


def _rows_into(case, k, v):
    """The case's cache holds rows k, v [tokens][H][D] of its one sequence."""
    from oracle import serving as os_

    where = [(0, t, int(case.table[0, t // case.P]), t % case.P) for t in range(int(case.lens[0]))]
    os_.append(case.cache, case.tag, case.P, where, case.bits(k), case.bits(v), case.dtype)


@pytest.mark.parametrize("apart", [8, 16, 20, 24, 30])
@pytest.mark.parametrize("tag,D", [(K8V8, 128), (K4V4, 64), (K8V4, 256)])
@pytest.mark.parametrize("dtype", [HALF, BF16])
@pytest.mark.parametrize("new", [1, 110])
def test_value_scales_far_apart(torch, tag, D, dtype, new, apart):
    """Every fourth token has values 2^apart times the others' and a score so low that it hardly counts: the
    others keep the precision they have by themselves."""
    from paper_2609_26219_amd import serving

    n = 200
    case = Case(93, tag, dtype, 1, 2, D, 16, (n,), (new,))
    rng = np.random.default_rng(apart)
    k, v, q = (rng.standard_normal(s) for s in ((n, 1, D), (n, 1, D), (new, 2, D)))
    large = np.arange(n) % 4 == 3
    q[:, :, 0], k[:, :, 0] = 30.0, np.where(large, -45.0, 0.0)[:, None]  # scores 84 and more below the others'
    top = 2.0 ** (12 if apart > 16 else 4)
    v *= np.where(large, top, top / 2.0 ** apart)[:, None, None]
    case.q = case.bits(q)
    _rows_into(case, k, v)
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
    _check_fine(case, out, lse)


@pytest.mark.parametrize("tag", [K8V8, K4V4])
@pytest.mark.parametrize("dtype", [HALF, BF16])
@pytest.mark.parametrize("new", [6, 110])
def test_value_scales_of_tokens_that_other_rows_see(torch, tag, dtype, new):
    """From one token on values are 2^24 times the earlier ones': rows before it, whose tile of tokens holds some, do not
    notice."""
    from paper_2609_26219_amd import serving

    n, first = 120, 117
    case = Case(94, tag, dtype, 1, 2, 128, 16, (n,), (new,))
    rng = np.random.default_rng(7)
    k, v = rng.standard_normal((n, 1, 128)), rng.standard_normal((n, 1, 128))
    v *= np.where(np.arange(n) >= first, 2.0 ** 12, 2.0 ** -12)[:, None, None]
    _rows_into(case, k, v)
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
    _check_fine(case, out, lse)


@pytest.mark.parametrize("tag", [FP16, K8V4, K4V4])
@pytest.mark.parametrize("equal", [True, False])
def test_rows_at_one_place(torch, tag, equal):
    """Equal rows at one place leave that row; rows that differ leave nothing in particular there, and every other place
    as it should be."""
    from oracle import serving as os_
    from paper_2609_26219_amd import serving

    n = 90
    case = Case(95, tag, BF16, 3, 1, 128, 16, (100,), (n,), scattered=True)
    case.positions[60:] = case.positions[:30][::-1]
    if equal:
        case.k[60:], case.v[60:] = case.k[:30][::-1], case.v[:30][::-1]
    cache, batch = _cache(torch, case), _batch(torch, case)
    serving.append(cache, batch, _up(torch, case.k, case), _up(torch, case.v, case))
    want = case.copy_of_cache()
    os_.append(want, tag, 16, case.where(), case.k, case.v, BF16)
    got, _ = _state(torch, cache, case)
    want = want["kv"] if tag == FP16 else [want["codes"], want["scales"]]
    twice = {(p, s) for _, _, p, s in case.where()[60:]}
    for g, w in zip(got, want):
        g = g.view(w.dtype)
        if not equal:  # those places aside
            for p, s in twice:
                for a in (g, w):
                    if tag == FP16:
                        a[p, s] = 0
                    elif a.ndim == 3:  # codes
                        at = 0
                        for bits in (wl.KEY_BITS[tag], wl.VALUE_BITS[tag]):
                            row = 128 * bits // 8
                            a[p, :, at + s * row:at + (s + 1) * row] = 0
                            at += 16 * row
                    else:
                        a[p, :, :, s] = 0
        assert np.array_equal(g, w)


@pytest.mark.parametrize("tag,dtype,D", [(FP16, HALF, 64), (FP16, BF16, 128), (FP16, HALF, 256), (K8V8, BF16, 128),
                                         (K8V4, HALF, 64), (K4V4, BF16, 256)])
@pytest.mark.parametrize("new", [1, 4, 60])
@pytest.mark.parametrize("P", [16, 4])
def test_infinities_and_nans_that_no_row_sees(torch, tag, dtype, D, new, P):
    """In few rows and many: behind the sinks and before every row's window, and past the end, in pages that rows do see."""
    from paper_2609_26219_amd import serving

    n, window, sinks = 150, 40, 5
    case = Case(97, tag, dtype, 1, 4, D, P, (n,), (new,))
    clean = case.copy_of_cache()
    nan = {HALF: 0x7E00, BF16: 0x7FC0}[dtype]
    inf = {HALF: 0x7C00, BF16: 0x7F80}[dtype]
    unseen = range(sinks, n - new + 1 - window)
    assert len(unseen) > 40
    for t in unseen:
        p, s = case.table[0, t // P], t % P
        if tag == FP16:
            for a in case.cache["kv"]:
                a[p, s] = (nan, inf, inf | 0x8000)[t % 3]
        else:
            case.cache["scales"][p, :, :, s] = (0x7E00, 0x7C00, 0xFC00)[t % 3]
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), window=window,
                                 sinks=sinks, return_lse=True)
    case.cache = clean
    check_attention(case, _down(out), lse.cpu().numpy(), window, sinks)


@pytest.mark.parametrize("tag", [FP16, K4V4])
@pytest.mark.parametrize("n,at", [(1, 0), (33, 32), (100, 99), (3000, 2999)])
def test_a_nan_that_a_row_sees_reaches_its_result(torch, tag, n, at):
    """Keys of one token are NaN, the only one in its tile of 32, its wave or its row: the result is NaN, not that of the
    other tokens (or, without others, of an empty row)."""
    from paper_2609_26219_amd import serving

    case = Case(98, tag, BF16, 1, 2, 64, 16, (n,), (1,))
    p, s = case.table[0, at // 16], at % 16
    if tag == FP16:
        case.cache["kv"][0][p, s] = 0x7FC0
    else:
        case.cache["scales"][p, :, 0, s] = 0x7E00
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    case.lens[0] = at  # up to that token
    if at:
        out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
        check_attention(case, _down(out), lse.cpu().numpy())


@pytest.mark.parametrize("dtype", [HALF, BF16])
@pytest.mark.parametrize("n", [60, 5000])
@pytest.mark.parametrize("new", [3, 45])
def test_a_row_that_sees_nothing_is_zero_whatever_others_see(torch, dtype, n, new):
    """Rows without a position beside rows that see infinite values."""
    from paper_2609_26219_amd import serving

    case = Case(99, FP16, dtype, 1, 1, 128, 16, (n,), (new,), scattered=True)
    case.positions[:] = n - 1
    case.positions[1::3] = -1
    case.cache["kv"][1][case.table[0, 1], 3] = {HALF: 0x7C00, BF16: 0x7F80}[dtype]
    out, lse = serving.attention(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case), return_lse=True)
    assert (out[1::3] == 0).all() and torch.isneginf(lse[1::3]).all()
    assert torch.isinf(out[0::3]).all() and torch.isfinite(lse[0::3]).all()


@pytest.mark.parametrize("tag", [FP16, K4V4])
@pytest.mark.parametrize("new", [2, 50])
def test_windows_and_sinks_past_every_sequence_cover_it(torch, tag, new):
    from paper_2609_26219_amd import serving

    case = Case(101, tag, BF16, 1, 2, 64, 16, (1500, 70), (new,))
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    want = serving.attention(cache, batch, q)
    check_attention(case, _down(want), case.attend()[1].astype(np.float32))
    for window, sinks in ((1 << 40, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 1 << 33), (1 << 32, 5)):
        out, lse = serving.attention(cache, batch, q, window=window, sinks=sinks, return_lse=True)
        check_attention(case, _down(out), lse.cpu().numpy())


@pytest.mark.parametrize("own_stream", [True, False])
def test_threads_on_one_cache(torch, own_stream):
    """Two host threads, each on a layer of its own (of one cache), on streams of their own or on one: every attention has
    the bits that it has alone."""
    import threading

    from paper_2609_26219_amd import serving

    case = Case(103, K4V4, BF16, 2, 4, 64, 16, (1500, 300), (1,), layers=2, layer=0)
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    cache.codes[1], cache.scales[1] = cache.codes[0].flip(-1), cache.scales[0] * 0.5
    want = [serving.attention(cache, batch, q, layer=layer) for layer in range(2)]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    results, errors = [[], []], []
    shared = torch.cuda.Stream()

    def work(layer):
        try:
            with torch.cuda.stream(torch.cuda.Stream() if own_stream else shared):
                for _ in range(40):
                    results[layer].append(serving.attention(cache, batch, q, layer=layer))
                torch.cuda.current_stream().synchronize()
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(layer,)) for layer in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and [len(r) for r in results] == [40, 40]
    for layer in range(2):
        assert all(torch.equal(r, want[layer]) for r in results[layer])


LEAST, MOST = -2 ** 31, 2 ** 31 - 1
GARBAGE = [
    # token_start, kv_lens of three sequences
    ([LEAST, 4, 4, MOST], [MOST, 0, MOST]),
    ([0, 4, 9, LEAST], [LEAST, MOST, 50]),
    ([3, LEAST, MOST, 7], [40, 50, LEAST]),
    ([MOST, LEAST, MOST, LEAST], [MOST, MOST, MOST]),
    ([-5, LEAST + 3, 6, 1 << 30], [-1, 1 << 30, 60]),
]


@pytest.mark.parametrize("starts,lens", GARBAGE)
@pytest.mark.parametrize("tag,group,width", [(FP16, 1, 10), (FP16, 8, 10), (K4V4, 2, 200), (K8V4, 16, 200), (FP16, 16, 300)])
@pytest.mark.parametrize("scattered", [False, True])
def test_device_arrays_of_any_contents_stay_within_the_buffers(torch, tag, group, width, starts, lens, scattered):
    """Starts, lengths, positions and page tables as memory that nobody has filled may hold them (the host cannot look):
    every call ends, writes its own rows alone, and the next call is right."""
    from paper_2609_26219_amd import serving

    case = Case(109, tag, BF16, 2, group, 64, 16, (70, 90, 130), (3, 4, 3), scattered=scattered, wide=width - 9)
    cache, batch = _cache(torch, case), _batch(torch, case, bounds=False)
    good = [None if t is None else t.clone() for t in batch.keep]
    fused = torch.full((case.tokens + 8, 2 * group + 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out, k, v = (fused[4:-4, a:b] for a, b in ((0, 2 * group), (2 * group, 2 * group + 2), (2 * group + 2, 2 * group + 4)))
    q = _up(torch, case.q, case)
    rng = np.random.default_rng(1)
    up = lambda a: torch.from_numpy(np.asarray(a, np.int64).astype(np.int32)).cuda()  # noqa: E731
    batch.keep[0].copy_(up(starts))
    batch.keep[1].copy_(up(lens))
    batch.keep[2].copy_(up(rng.choice([LEAST, -1, 0, 1, case.pool - 1, case.pool, MOST], case.table.shape)))
    if scattered:
        batch.keep[3].copy_(up(rng.choice([LEAST, -1, 0, 5, 159, 1 << 30, MOST], case.tokens)))
    for window, sinks in ((0, 0), (20, 3)):
        serving.attention(cache, batch, q, out=out, window=window, sinks=sinks, return_lse=True)
    serving.read(cache, batch, out=(k, v))
    torch.cuda.synchronize()
    assert (fused[:4] == 7.0).all() and (fused[-4:] == 7.0).all()
    for t, g in zip(batch.keep, good):
        if t is not None:
            t.copy_(g)
    got, lse = serving.attention(cache, batch, q, return_lse=True)
    check_attention(case, _down(got), lse.cpu().numpy())
