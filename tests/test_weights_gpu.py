"""The attention weight that cached tokens receive, on the GPU against the fp64 oracle: few rows and many, all cache types,
masks that leave rows and tokens empty, pages that are not there."""
import numpy as np
import pytest

from oracle import serving as os_
from paper_2609_26219_amd import binding as pb
from serving_cases import Case
from test_serving_gpu import _batch, _cache, _up

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


def _check(case, got, before, decay, joint, lse, window=0, sinks=0, scale=None):
    """Each weight within its derived bound.  An exponential's argument carries the score's error, 2^-23 (D / 8 + 16) of the
    reach scale * sum |q| (|k - zero| + |zero|) (single-precision sums of D products and the roundings around them), and 2^-22
    of |score| + |lse| from the products with log2 e and their difference; the exponential itself 2^-21.  A sum of n
    of them rounds n times, the decayed weight twice."""
    scale = case.D ** -0.5 if scale is None else scale
    want, slack, terms = os_.weigh(case.cache, case.tag, case.P, case.dtype, case.where(), case.lens, case.table, case.pool,
                                   case.q, lse, case.H, scale, window, sinks)
    tol = slack * 2.0 ** -23 * (case.D / 8 + 18) + want * (2.0 ** -21 + terms * 2.0 ** -24)
    if joint:
        want, tol, terms = (a.sum(1, keepdims=True) for a in (want, tol, terms))
        tol = tol + want * case.H * 2.0 ** -24
    here = np.arange(want.shape[2]) < np.array(case.lens)[:, None, None]
    old = before[:, :, :want.shape[2]].astype(np.float64) if decay else np.zeros_like(want)
    d = float(np.float32(decay))
    want = want + d * old
    tol = tol + 2.0 ** -23 * np.abs(d * old) + 2.0 ** -24 * np.abs(want) + 2.0 ** -120
    off = np.abs(got[:, :, :want.shape[2]] - want)
    here = np.broadcast_to(here, off.shape)
    assert (off[here] <= tol[here]).all(), float((off[here] / tol[here]).max())
    assert (got[:, :, :want.shape[2]][~here] == 77.0).all() and (got[:, :, want.shape[2]:] == 77.0).all()


def _run(torch, case, joint, decay, window=0, sinks=0, scale=None, lse=None, in_place=False, bounds=True, wide=5):
    from paper_2609_26219_amd import serving

    cache, batch = _cache(torch, case), _batch(torch, case, bounds)
    q = _up(torch, case.q, case)
    if lse is None:
        _, lse = serving.attention(cache, batch, q, window=window, sinks=sinks, scale=scale, layer=case.layer,
                                   return_lse=True)
    rng = np.random.default_rng(1)
    tokens = (case.most_kv if bounds else case.table.shape[1] * case.P) + wide
    shape = (len(case.lens), 1 if joint else case.H, tokens)
    before = rng.exponential(1.0, shape).astype(np.float32)
    out = torch.full(shape, 77.0, device="cuda")
    if in_place:
        n = torch.tensor(case.lens, device="cuda")[:, None, None]
        out = torch.where(torch.arange(tokens, device="cuda") < n, torch.from_numpy(before).cuda(), out)
    got = serving.attention_weights(cache, batch, q, lse, out, out if in_place else
                                    (torch.from_numpy(before).cuda() if decay else None), decay=decay, scale=scale,
                                    window=window, sinks=sinks, layer=case.layer)
    assert got is out
    _check(case, out.cpu().numpy(), before, decay, joint, lse.cpu().numpy(), window, sinks, scale)
    return out


FEW = [
    # tag, dtype, H, group, D, P, lens, new
    (K4V4, BF16, 2, 4, 64, 16, (40, 3, 0, 17, 100), (1,)),
    (K4V4, HALF, 8, 4, 128, 16, (700, 1, 33), (1,)),
    (K8V4, BF16, 3, 5, 128, 1, (95, 31), (3, 2)),
    (K8V8, HALF, 1, 1, 256, 4, (130, 64), (7,)),
    (FP16, BF16, 8, 2, 128, 32, (257, 64, 5), (4,)),
    (FP16, HALF, 5, 8, 64, 8, (90,), (2,)),
    (FP16, BF16, 1, 16, 256, 64, (600,), (1,)),
    (K4V4, BF16, 12, 1, 64, 2, (50, 50), (32,)),
    (K8V8, BF16, 4, 16, 128, 16, (65,), (2,)),
    (FP16, HALF, 2, 16, 128, 16, (300, 45), (2,)),
    (FP16, BF16, 2, 16, 64, 4, (70, 45), (2,)),
]
MANY = [
    (K4V4, BF16, 2, 4, 64, 16, (40, 3, 0, 300), (40, 3, 1, 50)),
    (K8V4, HALF, 1, 5, 128, 1, (95, 31), (33, 31)),
    (K8V8, BF16, 2, 1, 256, 4, (200, 64), (130, 64)),
    (FP16, BF16, 2, 2, 128, 32, (515, 64, 5), (64, 64, 5)),
    (FP16, HALF, 3, 8, 64, 8, (90,), (90,)),
    (FP16, BF16, 1, 3, 256, 64, (140,), (20,)),
    (K4V4, HALF, 1, 4, 128, 16, (300,), (300,)),
    (FP16, HALF, 1, 4, 128, 16, (1, 270), (1, 270)),
]


@pytest.mark.parametrize("tag,dtype,H,group,D,P,lens,new", FEW + MANY)
@pytest.mark.parametrize("joint", [False, True])
def test_weights(torch, tag, dtype, H, group, D, P, lens, new, joint):
    case = Case(21 + D + H, tag, dtype, H, group, D, P, lens, new, holes=1, layers=2, layer=1)
    _run(torch, case, joint, decay=0.75)


@pytest.mark.parametrize("tag,dtype,H,group,D,P,lens,new", FEW + MANY)
@pytest.mark.parametrize("window,sinks", [(1, 0), (37, 0), (16, 5), (100, 40)])
def test_weights_with_a_window(torch, tag, dtype, H, group, D, P, lens, new, window, sinks):
    case = Case(22 + D + H, tag, dtype, H, group, D, P, lens, new)
    _run(torch, case, joint=True, decay=0.0, window=window, sinks=sinks)


@pytest.mark.parametrize("tag,dtype,H,group,D,P,lens,new", FEW[::2] + MANY[::2])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_weights_of_scattered_rows(torch, tag, dtype, H, group, D, P, lens, new, window, sinks):
    """Rows anywhere, some past kv_lens or at a negative position, in no order."""
    case = Case(23 + D + H, tag, dtype, H, group, D, P, lens, new, scattered=True, holes=1)
    case.positions[::5] = -1
    case.positions[2::7] = case.most_kv + 9
    _run(torch, case, joint=False, decay=1.0, window=window, sinks=sinks, in_place=True)


def test_weights_without_bounds(torch):
    """max_tokens and max_kv_len unknown: the launch goes by the table and the number of rows."""
    for new in ((1,), (30,)):
        case = Case(24, K4V4, BF16, 2, 2, 64, 16, (40, 33), new, wide=3)
        _run(torch, case, joint=False, decay=1.0, bounds=False)


@pytest.mark.parametrize("tag,dtype,D,group,joint", [(FP16, BF16, 64, 16, False), (K4V4, HALF, 128, 8, True),
                                                     (K8V4, BF16, 256, 9, False), (FP16, HALF, 128, 7, True)])
def test_many_rows_in_splits(torch, tag, dtype, D, group, joint):
    """So many rows that several workgroups share a tile of tokens, whose parts are joined."""
    case = Case(40 + D, tag, dtype, 1, group, D, 16, (330, 290), (330, 9))
    _run(torch, case, joint=joint, decay=0.5)
    _run(torch, case, joint=joint, decay=1.0, window=33, sinks=3, in_place=True)


@pytest.mark.parametrize("H,joint", [(1, False), (2, True), (3, False), (5, True)])
def test_shares_of_ragged_sequences_added_in_place(torch, H, joint):
    """Workgroups' even shares end inside sequences and inside their waves' parts: every token is added to once."""
    lens = tuple(int(n) for n in np.random.default_rng(H).integers(0, 400, 37)) + (0, 1, 33, 1000)
    case = Case(35 + H, K4V4, BF16, H, 2, 64, 16, lens, (1,))
    _run(torch, case, joint=joint, decay=1.0, in_place=True)


def test_more_sequences_than_are_shared(torch):
    lens = tuple(int(n) for n in np.random.default_rng(9).integers(0, 20, 530))
    case = Case(39, K4V4, HALF, 1, 1, 64, 16, lens, (1,))
    _run(torch, case, joint=True, decay=1.0, in_place=True)


@pytest.mark.parametrize("tag", [FP16, K8V4, K4V4])
@pytest.mark.parametrize("new", [(1,), (40,)])
def test_a_scale_of_its_own_and_large_scores(torch, tag, new):
    """Scores of a hundred and more, where an exponential without the log-sum-exp would overflow."""
    case = Case(25, tag, BF16, 2, 3, 64, 16, (70,), new, scale_of_values=2.0)
    _run(torch, case, joint=False, decay=0.5, scale=0.5)


@pytest.mark.parametrize("new", [(1,), (40,)])
def test_rows_that_saw_nothing_give_nothing(torch, new):
    """A row whose lse is -inf adds nothing, whatever it could see; every page of one sequence is not there."""
    case = Case(26, K4V4, HALF, 2, 2, 64, 16, (60, 60), new)
    case.table[1] = -1
    lse = np.random.default_rng(0).normal(4.0, 1.0, (case.tokens, 4)).astype(np.float32)
    lse[::3, 1] = -np.inf
    _run(torch, case, joint=False, decay=1.0, lse=torch.from_numpy(lse).cuda())


@pytest.mark.parametrize("new", [(1,), (40,)])
@pytest.mark.parametrize("tag", [FP16, K4V4])
def test_weights_sum_to_the_number_of_rows(torch, tag, new):
    """Every query row deals out 1: the weights of a sequence add up to its rows times query heads."""
    from paper_2609_26219_amd import serving

    case = Case(27, tag, BF16, 2, 4, 128, 16, (500, 77), new)
    out = _run(torch, case, joint=True, decay=0.0)
    sums = torch.where(out == 77.0, 0.0, out).double().sum((1, 2)).cpu().numpy()
    assert np.abs(sums - np.diff(case.start) * 8).max() <= 1e-3 * np.diff(case.start).max() * 8
    assert serving is not None


@pytest.mark.parametrize("new", [(1,), (40,)])
@pytest.mark.parametrize("tag", [FP16, K4V4])
def test_garbage_that_no_row_sees(torch, tag, new):
    """NaN before every row's window and behind the sinks, and in keys of other tokens' pages: the cache's poison stays."""
    case = Case(28, tag, BF16, 1, 2, 64, 16, (90,), new)
    cached = case.cache
    for t in range(8, 90 - new[0] - 20):  # between the sinks and the earliest window
        p, slot = case.table[0, t // 16], t % 16
        if tag == FP16:
            cached["kv"][0][p, slot] = 0x7FC0
        else:
            cached["scales"][p, :, 0, slot] = 0x7E00
    out = _run(torch, case, joint=False, decay=0.0, window=20, sinks=8)
    assert not out.isnan().any()


@pytest.mark.parametrize("new", [(1,), (40,)])
def test_a_nan_key_reaches_its_own_weight_only(torch, new):
    from paper_2609_26219_amd import serving

    case = Case(29, FP16, BF16, 1, 2, 64, 16, (90,), new)
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    _, lse = serving.attention(cache, batch, q, return_lse=True)
    out = torch.empty((1, 1, 90), device="cuda")
    serving.attention_weights(cache, batch, q, lse, out)
    cache.k_cache[case.layer, int(case.table[0, 2]), 3] = float("nan") if cache.k_cache.dtype == torch.bfloat16 else 0x7FC0
    bad = serving.attention_weights(cache, batch, q, lse, torch.empty_like(out))
    keep = torch.arange(90, device="cuda") != 35
    assert bad[0, 0, 35].isnan() and torch.equal(bad[0, 0, keep], out[0, 0, keep])


def test_no_rows_only_fade(torch):
    from paper_2609_26219_amd import serving

    case = Case(30, K4V4, BF16, 2, 2, 64, 16, (20, 7), (1,))
    cache = _cache(torch, case)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = serving.Batch(dev([0, 0, 0]), dev([20, 7]), dev(case.table), 0, max_kv_len=20)
    w = torch.rand((2, 2, 20), device="cuda")
    out = torch.full_like(w, 3.0)
    serving.attention_weights(cache, batch, torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"),
                              torch.empty((0, 4), device="cuda"), out, w, decay=0.5)
    here = torch.arange(20, device="cuda") < torch.tensor([20, 7], device="cuda")[:, None, None]
    assert torch.equal(out, torch.where(here, 0.5 * w, 3.0))


@pytest.mark.parametrize("new,joint", [((1,), True), ((60,), True), ((60,), False)])
def test_calls_repeat_bit_for_bit_and_in_graphs(torch, new, joint):
    """Two graphs with workspaces of their own, replayed in turn with eager calls between, as lengths and queries change."""
    from paper_2609_26219_amd import serving

    cases = [Case(31 + i, K4V4, BF16, 4, 4, 64, 16, (200, 90), new) for i in range(2)]
    made = []
    for case in cases:
        cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
        out = torch.zeros((2, 1 if joint else 4, 200), device="cuda")

        def step(cache=cache, batch=batch, q=q, out=out):
            _, lse = serving.attention(cache, batch, q, return_lse=True)
            return serving.attention_weights(cache, batch, q, lse, out, out, decay=0.5)

        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        made.append((batch, q, out, step, graph))
    for i in range(6):
        batch, q, out, step, graph = made[i % 2]
        q.copy_(torch.randn_like(q))
        batch.keep[1].sub_(1)
        before = out.clone()
        graph.replay()
        made[1 - i % 2][4].replay()
        got = out.clone()
        out.copy_(before)
        step()
        assert torch.equal(got, out)


def test_streams_of_their_own(torch):
    """Calls on two streams have workspaces of their own."""
    from paper_2609_26219_amd import serving

    case = Case(33, FP16, BF16, 2, 4, 64, 16, (250,), (60,))
    cache, batch = _cache(torch, case), _batch(torch, case)
    qs = [_up(torch, case.q, case), torch.randn((60, 8, 64), device="cuda").bfloat16()]
    want = []
    for q in qs:
        _, lse = serving.attention(cache, batch, q, return_lse=True)
        want.append((lse, serving.attention_weights(cache, batch, q, lse, torch.empty((1, 1, 250), device="cuda"))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [torch.empty((1, 1, 250), device="cuda") for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, (lse, _), out, stream in zip(qs, want, got, streams):
            with torch.cuda.stream(stream):
                serving.attention_weights(cache, batch, q, lse, out)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, (_, w) in zip(got, want))


def test_refusals(torch):
    from paper_2609_26219_amd import serving

    case = Case(34, K4V4, BF16, 2, 2, 64, 16, (20, 9), (2, 1))
    cache, batch, q = _cache(torch, case), _batch(torch, case), _up(torch, case.q, case)
    lse, out = torch.zeros((3, 4), device="cuda"), torch.zeros((2, 2, 20), device="cuda")
    bad = [dict(lse=lse[:2]), dict(lse=lse.half()), dict(lse=lse.t().contiguous().t()), dict(out=out.double()),
           dict(out=out[:1]), dict(out=torch.zeros((2, 3, 20), device="cuda")), dict(out=out.transpose(1, 2)),
           dict(weights=torch.zeros((2, 2, 24), device="cuda")), dict(weights=torch.zeros((2, 2, 24), device="cuda")[..., :20])]
    for kw in bad:
        with pytest.raises(ValueError):
            serving.attention_weights(cache, batch, q, **{**dict(lse=lse, out=out), **kw})
    for kw in (dict(out=out[..., :19]), dict(out=out.cpu()), dict(decay=float("nan"), weights=out), dict(scale=0.0), dict(scale=1e-30),
               dict(window=-1), dict(sinks=-1), dict(layer=1)):
        with pytest.raises(pb.PkvError):
            serving.attention_weights(cache, batch, q, **{**dict(lse=lse, out=out), **kw})


INFINITE = [
    # dtype, H, group, D, P, lens, new: rows of a KV head that are part of a tile, a tile and part of one, two; many
    (BF16, 2, 4, 128, 16, (75,), (1,)),
    (HALF, 2, 5, 64, 16, (75, 40), (1,)),
    (BF16, 1, 3, 256, 1, (75,), (1,)),
    (HALF, 1, 1, 128, 32, (600,), (1,)),
    (BF16, 2, 6, 64, 8, (75,), (3,)),
    (HALF, 3, 8, 128, 16, (100,), (4,)),
    (BF16, 1, 3, 128, 16, (300,), (40,)),
    (HALF, 2, 4, 64, 4, (300, 290), (40, 37)),
    (BF16, 1, 2, 256, 16, (200,), (50,)),
]


@pytest.mark.parametrize("dtype,H,group,D,P,lens,new", INFINITE)
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 4)])
@pytest.mark.parametrize("value", [-np.inf, np.inf])
@pytest.mark.parametrize("mixed", [False, True])
def test_an_infinite_key_weighs_what_its_scores_say(torch, dtype, H, group, D, P, lens, new, window, sinks, value, mixed):
    """A channel of some keys is infinite, so every score there is too: -inf adds nothing, +inf makes the weight infinite,
    wherever the token lies in its tile and however many rows there are.  Other tokens' weights keep their bits."""
    from paper_2609_26219_amd import serving

    case = Case(36 + D, FP16, dtype, H, group, D, P, lens, new)
    rng = np.random.default_rng(D + H)
    channel, sign = 13, 0x8000
    if not mixed:
        case.q[:, :, channel] &= 0x7FFF
    case.q[:, :, channel] |= 0x2000  # (not zero, and of 2 and more so large that finite keys' scores overflow as well)
    lse = rng.normal(4.0, 1.0, (case.tokens, H * group)).astype(np.float32)
    before = rng.exponential(1.0, (len(lens), H, max(lens))).astype(np.float32)
    q, dlse, dbefore = _up(torch, case.q, case), torch.from_numpy(lse).cuda(), torch.from_numpy(before).cuda()
    batch = _batch(torch, case)

    def weigh():
        return serving.attention_weights(_cache(torch, case), batch, q, dlse, torch.full_like(dbefore, 77.0), dbefore, decay=0.75,
                                         window=window, sinks=sinks).cpu().numpy()

    finite = weigh()
    bad = np.zeros((len(lens), max(lens)), bool)
    infinite = {HALF: 0x7C00, BF16: 0x7F80}[dtype] | (sign if value < 0 else 0)
    for s, n in enumerate(lens):
        for t in (1, 17, n // 2, n - 33, n - 2, n - 1):
            bad[s, t] = True
            case.cache["kv"][0][case.table[s, t // P], t % P, :, channel] = infinite
    got = weigh()
    with np.errstate(all="ignore"):
        want, _, _ = os_.weigh(case.cache, FP16, P, dtype, case.where(), case.lens, case.table, case.pool, case.q, lse, H,
                               D ** -0.5, window, sinks)
        want = (want + 0.75 * before).astype(np.float32)
    for s in range(len(lens)):
        assert np.array_equal(got[s][:, bad[s]], want[s][:, bad[s]])
        assert np.array_equal(got[s][:, ~bad[s]], finite[s][:, ~bad[s]])
    assert not np.isnan(got).any()
    reached = np.concatenate([want[s][:, bad[s]].ravel() for s in range(len(lens))])
    assert mixed or np.isinf(reached).any() == (value > 0)
