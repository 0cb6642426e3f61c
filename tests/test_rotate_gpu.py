"""Rows turned to their rotary positions on the GPU, against the fp64 oracle, and turned on their way into the cache,
against the two calls one after the other, bit for bit."""
import numpy as np
import pytest

from oracle import serving as os_
from oracle.quantize import cache_values
from paper_2609_26219_amd import binding as pb
from paper_2609_26219_amd import workloads as wl
from serving_cases import UNIT, Case
from test_serving_gpu import _batch, _cache, _down, _dtype, _state, _up

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


def _with_rope(torch, case, style, rotary, freq, amplitude):
    """The case's cache with a RoPE of its own."""
    from paper_2609_26219_amd import serving
    plain = _cache(torch, case)
    kw = dict(num_kv_heads=case.H, head_dim=case.D, page_size=case.P, dtype=_dtype(torch, case), tag=case.tag,
              rope_style=style, rotary_dim=rotary, inv_freq=freq, rope_amplitude=amplitude)
    if case.tag == FP16:
        return serving.PagedCache(k_cache=plain.k_cache, v_cache=plain.v_cache, **kw)
    return serving.PagedCache(codes=plain.codes, scales=plain.scales, **kw)


def _check(case, have_bits, x_bits, offset, freq, style, amplitude):
    """Each element is the exact value rounded to single precision and then to the output type, half a step and 2^-9 of it;
    the angle's cosine and sine and the products are off by less than 2^-50 of |x| + |y| (four roundings of 2^-53)."""
    x = cache_values(x_bits, case.dtype)
    amplitude = float(np.float32(amplitude))
    want = os_.rotate(x, case.where(), offset, freq, style, amplitude)
    have = cache_values(have_bits, case.dtype)
    size = os_.rotate(np.abs(x), [(s, 0 if p >= 0 else p, *r) for s, p, *r in case.where()], np.zeros(len(case.lens)),
                      np.zeros(len(freq)), style, 1.0)  # |x| as it lies
    n = 2 * len(freq)
    pair = size.copy()
    if style:
        pair[..., 0:n:2] = pair[..., 1:n:2] = size[..., 0:n:2] + size[..., 1:n:2]
    else:
        pair[..., :n // 2] = pair[..., n // 2:n] = size[..., :n // 2] + size[..., n // 2:n]
    tol = np.abs(want) * UNIT[case.dtype] * (1 + 2.0 ** -9) + 2.0 ** -50 * max(1.0, abs(amplitude)) * pair + \
        (2.0 ** -25 if case.dtype == HALF else 0.0)
    off = np.abs(have - want)
    assert (off <= tol).all(), float((off / np.maximum(tol, 1e-300)).max())


SHAPES = [
    # dtype, D, rotary, style, heads, lens, new, far, amplitude
    (BF16, 128, 0, 0, 32, (7, 1, 0, 40), (1,), 0, 1.0),
    (HALF, 128, 64, 1, 5, (33, 20), (33, 7), 100000, 1.25),
    (HALF, 64, 16, 0, 1, (3,), (3,), 5, 0.5),
    (BF16, 256, 128, 1, 3, (70,), (70,), 1 << 29, 1.0),
    (BF16, 96, 96, 0, 7, (9, 5), (9, 2), -3, 1.0),
    (HALF, 96, 48, 1, 7, (9, 5), (9, 2), 1 << 20, 1.0),
    (HALF, 16, 16, 1, 40, (300,), (300,), 12345, 1.1),
    (BF16, 512, 512, 0, 2, (11,), (11,), 1, 1.0),
    (BF16, 80, 32, 0, 9, (150, 151), (150, 149), 77, 1.0),
]


@pytest.mark.parametrize("dtype,D,rotary,style,heads,lens,new,far,amplitude", SHAPES)
@pytest.mark.parametrize("scattered", [False, True])
def test_rotate_is_the_definition(torch, dtype, D, rotary, style, heads, lens, new, far, amplitude, scattered):
    from paper_2609_26219_amd import serving

    case = Case(7 + D + heads, K4V4, dtype, 1, heads, D, 16, lens, new, scattered=scattered)
    n = (rotary or D) // 2
    freq = [5e5 ** (-j / n) for j in range(n)]
    cache, batch = _with_rope(torch, case, style, rotary, freq, amplitude), _batch(torch, case)
    offset = np.array([far // (1 + s) for s in range(len(lens))], np.int32)
    q = _up(torch, case.q, case)
    out = serving.rotate(cache, batch, q, position_offset=torch.from_numpy(offset).cuda())
    assert np.array_equal(_down(q), case.q)
    _check(case, _down(out), case.q, offset, freq, style, amplitude)
    assert serving.rotate(cache, batch, q, out=q, position_offset=torch.from_numpy(offset).cuda()) is q
    assert np.array_equal(_down(q), _down(out))


def test_frequencies_from_theta_and_scaled(torch):
    """Without a table theta gives the frequencies; a table as for long contexts is taken as it is."""
    from paper_2609_26219_amd import serving

    case = Case(1, K8V8, BF16, 2, 2, 128, 16, (600, 40), (600, 40))
    freq = [10000.0 ** (-j / 64) for j in range(64)]
    out = serving.rotate(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case))
    _check(case, _down(out), case.q, np.zeros(2), freq, 0, 1.0)
    freq = wl.llama3_inv_freq(5e5, 128)
    cache = _with_rope(torch, case, 0, 0, freq, 1.0)
    out = serving.rotate(cache, _batch(torch, case), _up(torch, case.q, case))
    _check(case, _down(out), case.q, np.zeros(2), freq, 0, 1.0)


def test_position_zero_and_amplitude_one_copy(torch):
    """At position 0 the angle is 0, so that every element comes back bit for bit, whatever the type."""
    from paper_2609_26219_amd import serving
    for dtype in (HALF, BF16):
        case = Case(2, K4V4, dtype, 1, 3, 64, 16, (1,), (1,))
        out = serving.rotate(_cache(torch, case), _batch(torch, case), _up(torch, case.q, case))
        assert np.array_equal(_down(out), case.q)


def test_rows_of_no_sequence_stay_and_rows_without_a_position_are_copied(torch):
    from paper_2609_26219_amd import serving

    case = Case(3, K4V4, BF16, 1, 4, 64, 16, (10, 2, 5), (4, 4, 4))  # (the second sequence's first two rows are before it)
    cache, batch = _cache(torch, case), _batch(torch, case)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = serving.Batch(dev([1, 4, 8, 10]), dev(case.lens), dev(case.table), 12)
    out = torch.full((12, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = _up(torch, case.q, case)
    serving.rotate(cache, batch, q, out=out)
    got = _down(out)
    assert (_down(out[[0, 10, 11]]) == 0x40E0).all()
    assert np.array_equal(got[4:6], case.q[4:6])  # positions -2 and -1
    case.start = np.array([1, 4, 8, 10], np.int32)
    x = case.q.copy()
    x[[0, 10, 11]] = 0x40E0
    _check(case, got, x, np.zeros(3), [1e4 ** (-j / 32) for j in range(32)], 0, 1.0)


def test_infinities_and_nan_stay_in_their_pairs(torch):
    from paper_2609_26219_amd import serving

    case = Case(4, K4V4, BF16, 1, 2, 128, 16, (9,), (9,))
    cache = _with_rope(torch, case, 0, 64, [1e4 ** (-j / 32) for j in range(32)], 1.0)
    clean = serving.rotate(cache, _batch(torch, case), _up(torch, case.q, case))
    q = _up(torch, case.q, case)
    q[:, 0, 3], q[:, 1, 100] = float("nan"), float("inf")
    got = serving.rotate(cache, _batch(torch, case), q)
    assert got[:, 0, [3, 35]].isnan().all() and got[:, 1, 100].isinf().all()
    same = torch.ones((2, 128), dtype=torch.bool, device="cuda")
    same[0, [3, 35]] = same[1, 100] = False
    assert torch.equal(got[:, same], clean[:, same])


APPEND = [
    # tag, dtype, H, group, D, rotary, style, P, lens, new, far
    (K4V4, BF16, 8, 4, 128, 0, 0, 16, tuple(range(1, 41)), (1,), 99999),
    (K8V4, HALF, 3, 5, 128, 64, 1, 1, (9, 70), (9, 33), 7),
    (K8V8, BF16, 1, 1, 256, 64, 0, 4, (33, 1), (33, 1), 0),
    (K4V4, HALF, 5, 2, 96, 32, 1, 8, (21, 8, 0), (7,), 1 << 20),
    (K8V4, BF16, 2, 1, 16, 16, 0, 2, (130,), (130,), 3),
    (FP16, BF16, 2, 3, 128, 0, 0, 16, (31, 2), (9, 2), 50),
    (FP16, HALF, 3, 1, 48, 16, 1, 1, (5,), (5,), 0),
    (K8V8, HALF, 8, 8, 512, 512, 0, 32, (70,), (70,), 1),
]


@pytest.mark.parametrize("tag,dtype,H,group,D,rotary,style,P,lens,new,far", APPEND)
@pytest.mark.parametrize("scattered", [False, True])
def test_append_rotated_is_rotate_and_append(torch, tag, dtype, H, group, D, rotary, style, P, lens, new, far, scattered):
    """From views of one fused projection; codes, scales and rows bit for bit."""
    from paper_2609_26219_amd import serving

    case = Case(5 + D, tag, dtype, H, group, D, P, lens, new, scattered=scattered, holes=1)
    n = (rotary or D) // 2
    freq = [5e5 ** (-j / n) for j in range(n)]
    cache, batch = _with_rope(torch, case, style, rotary, freq, 1.125), _batch(torch, case)
    two = _with_rope(torch, case, style, rotary, freq, 1.125)
    offset = torch.tensor([far // (1 + s) for s in range(len(lens))], dtype=torch.int32, device="cuda")
    fused = torch.cat([_up(torch, t, case) for t in (case.q, case.k, case.v)], 1)
    q, k, v = fused.split([H * group, H, H], 1)
    got = serving.append_rotated(cache, batch, q, k, v, position_offset=offset)
    turned = serving.rotate(two, batch, k, position_offset=offset)
    serving.append(two, batch, turned, v.contiguous())
    assert torch.equal(got.view(torch.int16), serving.rotate(cache, batch, q, position_offset=offset).view(torch.int16))
    for a, b in zip(_state(torch, cache, case)[0], _state(torch, two, case)[0]):
        assert np.array_equal(a, b)
    _check(case, _down(turned), case.k, offset.cpu().numpy(), freq, style, 1.125)
    # in place, and the keys untouched
    again = serving.append_rotated(cache, batch, q, k, v, position_offset=offset, out=q)
    assert again is q and torch.equal(q.contiguous().view(torch.int16), got.view(torch.int16))
    assert np.array_equal(_down(k), case.k)


def test_many_rows_and_many_sequences(torch):
    """Token counts where a workgroup takes several tokens, and more sequences than starts fit LDS."""
    from paper_2609_26219_amd import serving

    S = 1500
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 90, S)
    case = Case(6, K4V4, HALF, 1, 2, 64, 16, tuple(int(n) for n in lens), (44,))
    freq = [1e4 ** (-j / 32) for j in range(32)]
    out = serving.rotate(_with_rope(torch, case, 0, 64, freq, 1.0), _batch(torch, case), _up(torch, case.q, case))
    assert case.tokens == 66000
    pick = rng.permutation(case.tokens)[:500]
    where = case.where()
    want = os_.rotate(cache_values(case.q[pick], HALF), [where[i] for i in pick], np.zeros(S), freq, 0, 1.0)
    have = cache_values(_down(out)[pick], HALF)
    assert (np.abs(have - want) <= np.abs(want) * 2.0 ** -11 * (1 + 2.0 ** -9) + 2.0 ** -25 + 2.0 ** -48).all()


def test_a_graph_follows_lengths_and_offsets(torch):
    from paper_2609_26219_amd import serving

    case = Case(8, K4V4, BF16, 2, 2, 64, 16, (20, 9), (1, 1))
    cache, batch = _cache(torch, case), _batch(torch, case)
    q, k, v = (_up(torch, t, case) for t in (case.q, case.k, case.v))
    offset = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    serving.append_rotated(cache, batch, q, k, v, out=out, position_offset=offset)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serving.append_rotated(cache, batch, q, k, v, out=out, position_offset=offset)
    for step in range(4):
        offset.add_(1000 * step)
        q.copy_(torch.randn_like(q))
        graph.replay()
        got = out.clone(), cache.codes.clone(), cache.scales.clone()
        cache.codes.zero_()
        eager = serving.append_rotated(cache, batch, q, k, v, position_offset=offset)
        assert torch.equal(got[0], eager)
        written = cache.codes != 0
        assert torch.equal(got[1][written], cache.codes[written]) and torch.equal(got[2].view(torch.int16),
                                                                                  cache.scales.view(torch.int16))


def test_refusals(torch):
    from paper_2609_26219_amd import serving

    case = Case(9, K4V4, BF16, 2, 2, 64, 16, (20, 9), (2, 1))
    cache, batch = _cache(torch, case), _batch(torch, case)
    q, k, v = (_up(torch, t, case) for t in (case.q, case.k, case.v))
    with pytest.raises(ValueError):
        serving.rotate(cache, batch, q[:2])
    with pytest.raises(ValueError):
        serving.rotate(cache, batch, q.half())
    with pytest.raises(ValueError):
        serving.rotate(cache, batch, q, position_offset=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        serving.rotate(cache, batch, q, position_offset=torch.zeros(2, device="cuda"))
    with pytest.raises(pb.PkvError):  # host memory
        serving.rotate(cache, batch, q, position_offset=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(pb.PkvError):
        serving.append_rotated(cache, batch, q, k, v, layer=3)
    for kw in (dict(rotary_dim=24), dict(rotary_dim=80), dict(rope_style=2), dict(inv_freq=[1.0]), dict(rope_theta=0.0),
               dict(rope_amplitude=float("nan")), dict(inv_freq=[float("inf")] * 32)):
        with pytest.raises(ValueError):
            serving.PagedCache(2, 64, 16, torch.bfloat16, K4V4, pool_pages=4, **kw)


def test_rotate_without_a_page_table(torch):
    from paper_2609_26219_amd import serving

    case = Case(77, K4V4, BF16, 2, 3, 64, 16, (20, 9), (4, 2))
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    want, out = serving.rotate(cache, batch, q), torch.empty_like(q)
    b = pb.PkvBatch.from_buffer_copy(batch.struct)
    b.page_table = None
    r = pb.PkvRotation(6, 1.0, None, q.data_ptr(), 6 * 64, 64, out.data_ptr(), 6 * 64, 64)
    assert pb.pkv_rotate_status(cache.model, b, r, torch.cuda.current_stream().cuda_stream) == pb.PKV_OK
    assert torch.equal(out, want)
