"""Host half of the eviction calls, without a GPU: refusals before any HIP call, sizes of workspaces, and the oracle's choice
and weights against other ways to work them out."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import serving as os_
from paper_2609_26219_amd import binding as pb
from serving_cases import Case
from test_serving_host import A, BAD, OK, TAG, _shape


def _call(which, shape=None, cache=None, batch=None, attention=None, weights=None, kept=None, table=(None, 0), drop=False):
    s = shape or _shape()
    m = pb.make_model(s)
    cb, sb = pb.pkv_cache_size(s, 3)
    c = pb.PkvPagedCache(**{**dict(tag=3, layer=1, codes=A, code_bytes=cb, scales=A, scale_bytes=sb), **(cache or {})})
    b = dict(num_seqs=0, num_tokens=0, max_tokens=0, pages_per_seq=4, max_kv_len=0, token_start=A, kv_lens=A,
             positions=None, page_table=A)
    b = pb.PkvBatch(**{**b, **(batch or {})})
    w = dict(heads=4, decay=1.0, tokens=64, head_stride=64, seq_stride=256, weights=A, out=A)
    w = pb.PkvWeights(**{**w, **(weights or {})})
    k = dict(heads=4, budget=16, sinks=2, recent=3, budgets=None, kept=A, kept_lens=A)
    k = pb.PkvKept(**{**k, **(kept or {})})
    if which == "weigh":
        a = dict(num_q_heads=8, window=0, sinks=0, scale=0.1, q=A, q_token_stride=1024, q_head_stride=128, out=None,
                 lse=A, workspace=A, workspace_bytes=1 << 40)
        return pb.pkv_attention_weights_status(m, c, b, pb.PkvAttention(**{**a, **(attention or {})}), w)
    if which == "keep":
        return pb.pkv_cache_keep_status(m, b, w, k)
    return pb.pkv_cache_evict_status(m, c, b, k, None if drop else w, *table)


EACH = pytest.mark.parametrize("which", ["weigh", "keep", "evict"])


@EACH
def test_nothing_to_do_is_ok(which):
    assert _call(which) == OK


@EACH
@pytest.mark.parametrize("batch", [dict(num_seqs=-1), dict(pages_per_seq=0), dict(max_kv_len=-1), dict(num_seqs=1 << 24),
                                   dict(num_seqs=1, kv_lens=None), dict(num_seqs=1, kv_lens=A + 2)])
def test_batch_refusals(which, batch):
    assert _call(which, batch=batch) == BAD


@EACH
@pytest.mark.parametrize("weights", [dict(heads=2), dict(heads=0), dict(tokens=63), dict(head_stride=63),
                                     dict(seq_stride=255), dict(weights=A + 2, out=A + 2), dict(weights=None, out=None),
                                     dict(tokens=1 << 41, head_stride=1 << 41, seq_stride=1 << 43)])
def test_weights_refusals(which, weights):
    assert _call(which, batch=dict(num_seqs=2), weights=weights) == BAD


def test_weights_are_not_needed_where_they_are_not_read():
    """A decay of zero reads none before; both only change what is checked after these (no GPU: a device error)."""
    ok = (OK, pb.PKV_ERR_DEVICE, BAD)  # with a GPU the address A is no device memory
    assert _call("weigh", batch=dict(num_seqs=2), weights=dict(weights=None)) == BAD
    assert _call("weigh", batch=dict(num_seqs=2), weights=dict(weights=None, decay=0.0)) in ok
    assert _call("evict", batch=dict(num_seqs=2), drop=True) in ok


@pytest.mark.parametrize("attention", [dict(num_q_heads=6), dict(window=-1), dict(sinks=-1), dict(scale=0.0),
                                       dict(scale=1e-30), dict(scale=float("nan")), dict(q=None), dict(q=A + 8), dict(lse=None),
                                       dict(lse=A + 2), dict(q_token_stride=3), dict(q_head_stride=64),
                                       dict(workspace=A + 8), dict(workspace_bytes=8)])
def test_attention_refusals(attention):
    assert _call("weigh", batch=dict(num_seqs=2, num_tokens=300), weights=dict(heads=4), attention=attention) == BAD


def test_weigh_refusals():
    assert _call("weigh", weights=dict(decay=float("nan"))) == BAD
    assert _call("weigh", weights=dict(decay=float("inf"))) == BAD
    assert _call("weigh", cache=dict(tag=4)) == TAG
    for dim in (16, 96, 192, 512):
        assert _call("weigh", shape=_shape(head_dim=dim)) == BAD
    big = dict(num_seqs=1 << 20, pages_per_seq=1 << 26)  # more workgroups than a launch has
    assert _call("weigh", batch=big, weights=dict(tokens=1 << 30, head_stride=1 << 30, seq_stride=1 << 32)) == BAD


@pytest.mark.parametrize("which", ["keep", "evict"])
@pytest.mark.parametrize("kept", [dict(heads=2), dict(heads=1), dict(budget=-1), dict(budget=(1 << 30) + 1),
                                  dict(sinks=-1), dict(recent=-1), dict(kept=None), dict(kept=A + 2),
                                  dict(kept_lens=None), dict(kept_lens=A + 1), dict(budgets=A + 3)])
def test_kept_refusals(which, kept):
    assert _call(which, batch=dict(num_seqs=2), kept=kept) == BAD


def test_evict_refusals():
    assert _call("evict", cache=dict(tag=-1)) == TAG
    assert _call("evict", cache=dict(layer=2)) == BAD
    assert _call("evict", table=(A, 0)) == BAD
    assert _call("evict", table=(A + 2, 4)) == BAD
    assert _call("evict", batch=dict(num_seqs=2, page_table=None)) == BAD
    assert _call("keep", batch=dict(num_seqs=1 << 23), kept=dict(heads=1), weights=dict(heads=1)) == BAD


def test_null_structures():
    lib, m, b, ref = pb.load(), pb.make_model(_shape()), pb.PkvBatch(pages_per_seq=4), ctypes.byref
    w, k = pb.PkvWeights(heads=1, tokens=64), pb.PkvKept(heads=1)
    assert lib.pkv_cache_keep(None, ref(b), ref(w), ref(k), None) == BAD
    assert lib.pkv_cache_keep(ref(m), None, ref(w), ref(k), None) == BAD
    assert lib.pkv_cache_keep(ref(m), ref(b), None, ref(k), None) == BAD
    assert lib.pkv_cache_keep(ref(m), ref(b), ref(w), None, None) == BAD
    assert lib.pkv_cache_evict(ref(m), None, ref(b), ref(k), None, None, 0, None) == BAD
    assert lib.pkv_attention_weights_workspace(ref(m), None, ref(b), None, ref(w), None) == BAD


def test_workspace():
    """None of few rows; of many the prepared rows, and sums of each head where they are joined."""
    s = _shape(pool_pages=4096)
    m, c = pb.make_model(s), pb.PkvPagedCache(tag=3)
    a = pb.PkvAttention(num_q_heads=16, scale=0.1)
    each = pb.PkvWeights(heads=4, tokens=65536, head_stride=65536, seq_stride=1 << 18)
    all_ = pb.PkvWeights(heads=1, tokens=65536, seq_stride=65536)
    one = pb.PkvBatch(num_seqs=3, num_tokens=3, max_tokens=1, pages_per_seq=4096)
    assert pb.pkv_attention_weights_workspace(m, c, one, a, each) == 0
    assert pb.pkv_attention_weights_workspace(m, c, one, a, all_) == 0
    many = pb.PkvBatch(num_seqs=3, num_tokens=192, max_tokens=64, pages_per_seq=4096)
    rows = (192 * 4 // 32 + 3 + 1) * 4 * (32 * (2 * 128 + 20) + 32)
    assert pb.pkv_attention_weights_workspace(m, c, many, a, each) == rows
    assert pb.pkv_attention_weights_workspace(m, c, many, a, all_) == rows + 3 * 4 * 65536 * 4


def test_rows_of_a_tile_stay_within_the_sequence(tmp_path):
    """The range of rows that a tile of tokens goes over, compiled for the host (weigh_rows_check.cpp)."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    here = os.path.dirname(os.path.abspath(__file__))
    root, exe = os.path.dirname(here), str(tmp_path / "check")
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-Wextra", "-I", os.path.join(root, "include"), "-I",
                    os.path.join(root, "paper_2609_26219_amd", "csrc"), os.path.join(here, "weigh_rows_check.cpp"), "-o",
                    exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout + run.stderr


def test_workspace_of_the_choice():
    """Few long rows are cut into segments, which need one."""
    m = pb.make_model(_shape())
    def nbytes(seqs, pages, heads=1):
        b = pb.PkvBatch(num_seqs=seqs, pages_per_seq=pages)
        tokens = pages * 16
        w = pb.PkvWeights(heads=heads, tokens=tokens, head_stride=tokens, seq_stride=heads * tokens)
        return pb.pkv_cache_keep_workspace(m, b, w, pb.PkvKept(heads=heads, budget=9))
    assert nbytes(1, 1536) == 0 and nbytes(65, 8192) == 0 and nbytes(0, 8192) == 0
    assert nbytes(3, 2049, 4) == 12 * 5 * (2048 * 4 + 8192 * 4 + 8) + 12 * 8
    assert _call("keep", batch=dict(num_seqs=1, pages_per_seq=4096), weights=dict(tokens=65536, head_stride=65536)) == BAD


def test_evict_to_the_same_table_of_another_width():
    assert _call("evict", batch=dict(num_seqs=2), table=(A, 3)) == BAD


def test_oracle_weights_are_column_sums():
    case = Case(5, 0, 0, 2, 3, 64, 8, (37, 9), (6, 9))
    _, lse, *_ = case.attend(window=11, sinks=2)
    lse32 = lse.astype(np.float32)
    w, _, _ = os_.weigh(case.cache, 0, 8, 0, case.where(), case.lens, case.table, case.pool, case.q, lse32, 2, 0.125, 11, 2)
    at = 0
    for s, (n, m) in enumerate(zip((37, 9), (6, 9))):
        k = np.stack([case.cache["kv"][0][case.table[s, t // 8], t % 8] for t in range(n)]).view(np.float16).astype(float)
        q = case.q[at:at + m].view(np.float16).astype(float)
        score = np.stack([q[:, h] @ k[:, h // 3].T for h in range(6)], 1) / 8.0  # [m, 6, n]
        pos, tok = np.arange(n - m, n)[:, None], np.arange(n)[None]
        score[~np.broadcast_to(((tok <= pos) & ((pos - tok < 11) | (tok < 2)))[:, None], score.shape)] = -np.inf
        p = np.exp(score - lse32[at:at + m, :, None].astype(float)).sum(0).reshape(2, 3, n).sum(1)
        assert np.allclose(w[s, :, :n], p, rtol=1e-12, atol=1e-300)
        at += m


def test_oracle_keep_by_hand():
    w = np.array([[[5, 1, 9, 3, 3, 7, 3, 0]], [[1, np.nan, 2, 0, 0, 0, 0, 0]]], np.float32)
    assert os_.keep(w, [8, 4], [5, 3], 1, 1) == [[[0, 2, 3, 5, 7]], [[0, 2, 3]]]
    assert os_.keep(w, [8, 0], [8, 3], 0, 0) == [[list(range(8))], [[]]]
    assert os_.keep(w, [8, 4], [2, 2], 5, 5) == [[[0, 1]], [[0, 1]]]
