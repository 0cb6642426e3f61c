"""What the eviction calls refuse and what they do not, on the host: each refusal beside the same call that passes every check
(without a GPU it ends at the device).  Every array has an address of its own."""
import pytest

from paper_2609_26219_amd import binding as pb
from test_serving_host import A, BAD, OK, _gpu_present, _shape

PASSES = pb.PKV_ERR_DEVICE

pytestmark = pytest.mark.skipif(_gpu_present(), reason="with a GPU these addresses are no device memory")


def _evict(num_seqs, shape, heads, budget, table=None, pages=4, tag=3, **kept):
    m = pb.make_model(shape)
    if tag:
        cb, sb = pb.pkv_cache_size(shape, tag)
        c = pb.PkvPagedCache(tag=tag, codes=A, code_bytes=cb, scales=2 * A, scale_bytes=sb)
    else:
        nbytes = 2 * shape.num_layers * shape.pool_pages * shape.page_size * shape.num_kv_heads * shape.head_dim
        c = pb.PkvPagedCache(tag=0, k_cache=A << 10, v_cache=A << 11, cache_bytes=nbytes)
    b = pb.PkvBatch(num_seqs, 0, 0, pages, 0, 3 * A, 4 * A, None, 5 * A)
    tokens = pages * shape.page_size
    w = pb.PkvWeights(heads, 1.0, tokens, tokens, heads * tokens, 6 * A, 6 * A)
    k = pb.PkvKept(**{**dict(heads=heads, budget=budget, kept=7 * A, kept_lens=8 * A), **kept})
    return pb.pkv_cache_evict_status(m, c, b, k, w, table, pages)


def test_launches_in_place_have_workgroups_of_1024_threads():
    """4 heads are 12 workgroups a sequence (weights, keys, values): below 2^22 in place and 2^24 to other pages."""
    most = ((1 << 22) - 1) // 12
    assert _evict(most, _shape(), 4, 9) == PASSES
    assert _evict(most + 1, _shape(), 4, 9) == BAD
    assert _evict(most + 1, _shape(), 4, 9, table=9 * A) == PASSES
    assert _evict(1 << 20, _shape(), 4, 9, table=9 * A) == BAD


@pytest.mark.parametrize("heads,dim", [(1, 32), (1, 16), (4, 128), (2, 256), (3, 48), (1, 512)])
@pytest.mark.parametrize("tag", range(4))
@pytest.mark.parametrize("budget", [0, 1, 100, 5000])
@pytest.mark.parametrize("table", [None, 9 * A])
def test_the_stated_bound_suffices(heads, dim, tag, budget, table):
    """num_seqs * num_kv_heads * ceil(head_dim / 32) * (3 + budget / 128) < 2^22."""
    shape = _shape(num_kv_heads=heads, head_dim=dim)
    per = heads * -(-dim // 32) * (3 * 128 + budget)
    seqs = ((1 << 22) * 128 - 1) // per
    assert seqs * per < (1 << 22) * 128
    assert _evict(seqs, shape, heads, budget, table, pages=512, tag=tag) == PASSES


def _keep(num_seqs=5, workspace=False, **kw):
    m = pb.make_model(_shape())
    at = {**dict(kv_lens=4 * A, budgets=9 * A, kept_lens=8 * A), **kw}
    b = pb.PkvBatch(num_seqs, 0, 0, 1 << 14 if workspace else 4, 0, 3 * A, at["kv_lens"], None, None)
    tokens = 16 << 14 if workspace else 64
    w = pb.PkvWeights(4, 1.0, tokens, tokens, 4 * tokens, 6 * A, None)
    k = pb.PkvKept(4, 16, 2, 3, at["budgets"], 7 * A, at["kept_lens"], 10 * A, 1 << 40)
    return pb.pkv_cache_keep_status(m, b, w, k)


@pytest.mark.parametrize("workspace", [False, True])
def test_the_choice_writes_none_of_what_it_reads(workspace):
    """Workgroups read lengths and budgets while others write kept_lens, so these lie apart."""
    assert _keep(workspace=workspace) == PASSES
    assert _keep(workspace=workspace, budgets=None) == PASSES
    for off in (0, 4, -4, 16, -16):
        assert _keep(workspace=workspace, kept_lens=4 * A + off) == BAD
        assert _keep(workspace=workspace, kept_lens=9 * A + off) == BAD
    for off in (20, -20):
        assert _keep(workspace=workspace, kept_lens=4 * A + off) == PASSES
        assert _keep(workspace=workspace, kept_lens=9 * A + off) == PASSES
    assert _keep(0, kept_lens=4 * A) == OK


def _weigh(decay, weights):
    m, s = pb.make_model(_shape()), _shape()
    cb, sb = pb.pkv_cache_size(s, 3)
    c = pb.PkvPagedCache(tag=3, codes=A, code_bytes=cb, scales=2 * A, scale_bytes=sb)
    b = pb.PkvBatch(2, 0, 0, 4, 0, 3 * A, 4 * A, None, 5 * A)
    a = pb.PkvAttention(num_q_heads=8, scale=0.1, q=6 * A, q_token_stride=1024, q_head_stride=128, lse=7 * A)
    w = pb.PkvWeights(4, decay, 64, 64, 256, weights, 8 * A)
    return pb.pkv_attention_weights_status(m, c, b, a, w)


def test_weights_before_are_needed_only_where_they_are_read():
    assert _weigh(0.5, 9 * A) == PASSES and _weigh(0.0, None) == PASSES
    assert _weigh(0.5, None) == BAD and _weigh(float("nan"), 9 * A) == BAD


def test_an_eviction_needs_no_weights():
    m, s = pb.make_model(_shape()), _shape()
    cb, sb = pb.pkv_cache_size(s, 3)
    c = pb.PkvPagedCache(tag=3, codes=A, code_bytes=cb, scales=2 * A, scale_bytes=sb)
    b = pb.PkvBatch(2, 0, 0, 4, 0, 3 * A, 4 * A, None, 5 * A)
    k = pb.PkvKept(heads=4, budget=16, kept=6 * A, kept_lens=7 * A)
    assert pb.pkv_cache_evict_status(m, c, b, k, None, None, 0) == PASSES
    for out, status in ((None, BAD), (8 * A + 2, BAD), (8 * A, PASSES)):
        assert pb.pkv_cache_evict_status(m, c, b, k, pb.PkvWeights(4, 1.0, 64, 64, 256, None, out), None, 0) == status


@pytest.mark.parametrize("kept", [dict(heads=2), dict(budget=-1), dict(budget=(1 << 30) + 1), dict(sinks=-1), dict(recent=-1),
                                  dict(kept=None), dict(kept=7 * A + 2), dict(kept_lens=None), dict(kept_lens=8 * A + 1),
                                  dict(budgets=9 * A + 3)])
def test_what_is_kept_is_refused_for_itself(kept):
    """The same call with nothing wrong passes, and with budget 0 it needs no place for the tokens."""
    def keep(**kw):
        m, b = pb.make_model(_shape()), pb.PkvBatch(2, 0, 0, 4, 0, 3 * A, 4 * A, None, None)
        w = pb.PkvWeights(4, 1.0, 64, 64, 256, 6 * A, None)
        at = dict(heads=4, budget=16, sinks=2, recent=3, budgets=9 * A, kept=7 * A, kept_lens=8 * A)
        return pb.pkv_cache_keep_status(m, b, w, pb.PkvKept(**{**at, **kw}))

    assert keep() == PASSES and keep(budget=0, kept=None) == PASSES
    assert keep(**kept) == BAD
