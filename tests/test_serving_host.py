"""Host half of the serving calls, without a GPU: sizes, refusals before any HIP call, and the oracle's attention against
a dense computation."""
import ctypes

import numpy as np
import pytest

from paper_2609_26219_amd import binding as pb
from paper_2609_26219_amd import workloads as wl
from serving_cases import Case

OK, BAD, TAG = pb.PKV_OK, pb.PKV_ERR_INVALID_ARGUMENT, pb.PKV_ERR_BAD_TAG


def _gpu_present():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:  # pragma: no cover
        return False


def _shape(**kw):
    base = dict(num_layers=2, num_kv_heads=4, head_dim=128, block_tokens=32, page_size=16, pool_pages=10,
                rope_theta=1e4, out_dtype=1)
    return wl.Shape(**{**base, **kw})


A = 1 << 20  # an aligned address that no call gets to use: every call below fails or has nothing to do


def _call(shape=None, cache=None, batch=None, attention=None, rows=None, which="attention"):
    s = shape or _shape()
    cb, sb = pb.pkv_cache_size(s, 3) if pb.load().pkv_cache_size(
        ctypes.byref(pb.make_model(s)), 3, ctypes.byref(ctypes.c_uint64()), ctypes.byref(ctypes.c_uint64())) == OK else (0, 0)
    c = dict(tag=3, layer=1, k_cache=None, v_cache=None, cache_bytes=0, codes=A, code_bytes=cb, scales=A, scale_bytes=sb)
    c.update(cache or {})
    b = dict(num_seqs=2, num_tokens=0, max_tokens=0, pages_per_seq=4, max_kv_len=0, token_start=A, kv_lens=A,
             positions=None, page_table=A)
    b.update(batch or {})
    m, c, b = pb.make_model(s), pb.PkvPagedCache(**c), pb.PkvBatch(**b)
    if which == "attention":
        a = dict(num_q_heads=8, window=0, sinks=0, scale=0.1, q=A, q_token_stride=1024, q_head_stride=128, out=A,
                 out_token_stride=1024, out_head_stride=128, lse=None, workspace=A, workspace_bytes=1 << 40)
        a.update(attention or {})
        return pb.pkv_attention_status(m, c, b, pb.PkvAttention(**a))
    r = dict(k=A, v=A, token_stride=512, head_stride=128)
    r.update(rows or {})
    f = pb.pkv_cache_append_status if which == "append" else pb.pkv_cache_read_status
    return f(m, c, b, r["k"], r["v"], r["token_stride"], r["head_stride"])


@pytest.mark.parametrize("which", ["attention", "append", "read"])
def test_nothing_to_do_is_ok(which):
    assert _call(which=which) == OK
    assert _call(which=which, batch=dict(num_seqs=0, num_tokens=5)) == OK


CACHE = [
    (dict(cache=dict(tag=4)), TAG), (dict(cache=dict(tag=-1)), TAG), (dict(cache=dict(layer=2)), BAD),
    (dict(cache=dict(layer=-1)), BAD), (dict(cache=dict(codes=None)), BAD), (dict(cache=dict(scales=None)), BAD),
    (dict(cache=dict(codes=A + 8)), BAD), (dict(cache=dict(scales=A + 4)), BAD), (dict(cache=dict(code_bytes=100)), BAD),
    (dict(cache=dict(scale_bytes=100)), BAD), (dict(cache=dict(tag=2)), BAD), (dict(cache=dict(tag=0)), BAD),
    (dict(cache=dict(tag=0, k_cache=A, v_cache=A + (1 << 30), cache_bytes=8)), BAD),
    (dict(cache=dict(tag=0, k_cache=A, v_cache=A, cache_bytes=1 << 30)), BAD),
    (dict(batch=dict(num_seqs=-1)), BAD), (dict(batch=dict(num_tokens=-1)), BAD), (dict(batch=dict(max_tokens=-1)), BAD),
    (dict(batch=dict(pages_per_seq=0)), BAD), (dict(batch=dict(max_kv_len=-1)), BAD),
    (dict(batch=dict(pages_per_seq=(1 << 26) + 1)), BAD),
    (dict(batch=dict(num_tokens=3, token_start=None)), BAD), (dict(batch=dict(num_tokens=3, kv_lens=None)), BAD),
    (dict(batch=dict(num_tokens=3, page_table=None)), BAD), (dict(batch=dict(num_tokens=3, kv_lens=A + 2)), BAD),
    (dict(batch=dict(num_tokens=3, positions=A + 1)), BAD),
    (dict(shape=_shape(page_size=12)), BAD), (dict(shape=_shape(num_layers=0)), BAD),
]


@pytest.mark.parametrize("kw,status", CACHE)
@pytest.mark.parametrize("which", ["attention", "append", "read"])
def test_cache_and_batch_refusals(kw, status, which):
    assert _call(which=which, **kw) == status


@pytest.mark.parametrize("rows", [dict(token_stride=4), dict(head_stride=64), dict(head_stride=132), dict(token_stride=-8),
                                  dict(k=A + 8), dict(v=A + 2), dict(k=None), dict(v=None)])
@pytest.mark.parametrize("which", ["append", "read"])
def test_row_refusals(rows, which):
    assert _call(which=which, batch=dict(num_tokens=1), rows=rows) == BAD


@pytest.mark.parametrize("attention", [dict(num_q_heads=6), dict(num_q_heads=0), dict(window=-1), dict(sinks=-1),
                                       dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                       dict(scale=float("inf")), dict(q=None), dict(out=None), dict(q=A + 8),
                                       dict(out=A + 2), dict(lse=A + 1), dict(q_token_stride=3), dict(out_head_stride=64),
                                       dict(workspace=None), dict(workspace_bytes=8), dict(workspace=A + 8)])
def test_attention_refusals(attention):
    kw = dict(batch=dict(num_tokens=2, max_tokens=1, pages_per_seq=1000), attention=attention)
    assert _call(**kw) == BAD


@pytest.mark.parametrize("dim", [16, 32, 96, 192, 512])
def test_attention_head_dims(dim):
    assert _call(shape=_shape(head_dim=dim)) == BAD


def test_too_many_rows_are_refused():
    assert _call(batch=dict(num_tokens=(1 << 28))) == BAD


@pytest.mark.parametrize("tag", range(4))
def test_sizes(tag):
    s = _shape(num_layers=3, head_dim=96, page_size=8, pool_pages=7)
    cb, sb = pb.pkv_cache_size(s, tag)
    rows = 3 * 7 * 8 * 4
    assert cb == (0 if tag == 0 else rows * 96 * (wl.KEY_BITS[tag] + wl.VALUE_BITS[tag]) // 8)
    assert sb == (0 if tag == 0 else rows * 8)
    lib = pb.load()
    out = ctypes.c_uint64()
    assert lib.pkv_cache_size(ctypes.byref(pb.make_model(s)), tag, None, ctypes.byref(out)) == BAD
    assert lib.pkv_cache_size(ctypes.byref(pb.make_model(s)), 9, ctypes.byref(out), ctypes.byref(out)) == TAG


def test_workspace_covers_few_rows_and_none_where_rows_fill_the_gpu():
    s = _shape(pool_pages=4096)
    m = pb.make_model(s)
    c = pb.PkvPagedCache(tag=3)
    a = pb.PkvAttention(num_q_heads=8, scale=0.1)
    few = pb.PkvBatch(num_seqs=1, num_tokens=1, max_tokens=1, pages_per_seq=4096)
    nbytes = pb.pkv_attention_workspace(m, c, few, a)
    per = 8 * (128 + 2) * 4
    assert nbytes > 0 and nbytes % per == 0 and nbytes // per <= 4096 * 16 // 32
    many = pb.PkvBatch(num_seqs=512, num_tokens=512 * 64, max_tokens=64, pages_per_seq=4096)
    assert pb.pkv_attention_workspace(m, c, many, a) == 0


def test_oracle_against_a_dense_computation():
    """The oracle's attention against softmax over whole rows built another way (16-bit cache, no unmapped pages)."""
    case = Case(5, 0, 0, 2, 3, 64, 8, (37, 9), (6, 9))
    out, lse, *_ = case.attend(window=11, sinks=2)
    at = 0
    for s, (n, m) in enumerate(zip((37, 9), (6, 9))):
        k, v = (np.stack([a[case.table[s, t // 8], t % 8] for t in range(n)]).view(np.float16).astype(np.float64)
                for a in case.cache["kv"])
        q = case.q[at:at + m].view(np.float16).astype(np.float64)
        score = np.einsum("ihd,thd->iht", q, np.repeat(k, 3, 1)) / 8.0
        pos, tok = np.arange(n - m, n)[:, None], np.arange(n)[None]
        ok = (tok <= pos) & ((pos - tok < 11) | (tok < 2))
        score[~np.broadcast_to(ok[:, None], score.shape)] = -np.inf
        w = np.exp(score)
        assert np.allclose(np.log(w.sum(-1)), lse[at:at + m], atol=1e-12)
        assert np.allclose(np.einsum("iht,thd->ihd", w / w.sum(-1, keepdims=True), np.repeat(v, 3, 1)), out[at:at + m],
                           atol=1e-12)
        at += m


def test_oracle_rows_by_hand():
    """A row 0, 1, .. 15 in 4 bits: zero 0, scale 1, codes the values; nibbles low first."""
    from oracle import serving as os_
    codes, scale, zero = os_.quantise_row(np.arange(16.0), 4)
    assert (scale, zero) == (1.0, 0.0) and list(codes) == list(range(16))
    cache = {"codes": np.zeros((1, 1, 32), np.uint8), "scales": np.zeros((1, 1, 2, 2, 2), np.uint16)}
    bits = np.arange(16, dtype=np.float16).view(np.uint16)[None, None]
    os_.append(cache, 3, 2, [(0, 1, 0, 1)], bits, bits, 0)
    assert list(cache["codes"][0, 0, 8:16]) == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    assert list(cache["codes"][0, 0, 24:32]) == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    assert not cache["codes"][0, 0, :8].any() and not cache["codes"][0, 0, 16:24].any()
    assert cache["scales"][0, 0, 0, 1, 0] == 0x3C00 and cache["scales"][0, 0, 0, 0, 0] == 0
    x, free, mid = os_.row(cache, 3, 2, 0, 0, 0, 1, 0)
    assert list(x) == list(range(16)) and list(free) == [abs(i - 8) for i in range(16)] and mid == 8.0


def test_sizes_past_a_launch_are_refused():
    """2^24 sequences, rows or workgroups, and pages whose stride passes 32 bits."""
    for which in ("attention", "append", "read"):
        assert _call(which=which, batch=dict(num_seqs=1 << 24)) == BAD
        assert _call(which=which, batch=dict(num_tokens=1 << 24)) == BAD
    assert _call(batch=dict(num_tokens=1 << 21, max_tokens=1, pages_per_seq=1000)) == BAD  # 2^24 rows to join
    assert _call(batch=dict(num_seqs=1 << 20, num_tokens=1 << 20, max_tokens=1024)) == BAD  # 2^27 workgroups
    s = _shape(num_layers=1, num_kv_heads=8, head_dim=128, page_size=1 << 20, pool_pages=2)
    m, b, a = pb.make_model(s), pb.PkvBatch(num_seqs=1, num_tokens=1, pages_per_seq=1), pb.PkvAttention(num_q_heads=8, scale=1.0)
    for paired, ok in ((0, True), (1, False)):  # 2 GiB of keys; keys and values on one page
        m.kv_layout = paired
        if ok:
            pb.pkv_attention_workspace(m, pb.PkvPagedCache(tag=0), b, a)
        else:
            with pytest.raises(pb.PkvError):
                pb.pkv_attention_workspace(m, pb.PkvPagedCache(tag=0), b, a)
        pb.pkv_attention_workspace(m, pb.PkvPagedCache(tag=3), b, a)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tag", range(4))
@pytest.mark.parametrize("empty", [dict(num_tokens=0), dict(num_seqs=0, num_tokens=3), dict(num_seqs=0, num_tokens=0)])
def test_an_empty_batch_needs_nothing_however_long_its_sequences_may_be(dim, tag, empty):
    """No row, or no sequence, over page tables of 16000 tokens: nothing to launch and no workspace."""
    s = _shape(head_dim=dim)
    m, c = pb.make_model(s), pb.PkvPagedCache(tag=tag)
    for group in (1, 2, 40):
        b = pb.PkvBatch(**{**dict(num_seqs=2, max_tokens=0, pages_per_seq=1000), **empty})
        a = pb.PkvAttention(num_q_heads=4 * group, scale=0.1)
        assert pb.pkv_attention_workspace(m, c, b, a) == 0
    if tag == 3:  # (the codes that _call describes)
        assert _call(shape=s, batch=dict(pages_per_seq=1000, **empty),
                     attention=dict(q_head_stride=dim, out_head_stride=dim, workspace=None, workspace_bytes=0)) == OK


def test_the_bound_of_a_launch_that_always_suffices():
    """(num_seqs + 1) * heads * ceil(max_tokens * group / 16) < 2^23, over every form: sizes right below it are taken."""
    rng = np.random.default_rng(1)
    lib, taken = pb.load(), 0
    for _ in range(4000):
        dim, tag, heads = int(rng.choice([64, 128, 256])), int(rng.integers(4)), int(2 ** rng.uniform(0, 7))
        group, most = int(2 ** rng.uniform(0, 6)), int(2 ** rng.uniform(0, 12))
        if heads * dim > 4096:  # (a row of the model)
            continue
        per = heads * -(-most * group // 16)
        seqs = ((1 << 23) - 1) // per - 1 - int(rng.integers(3))
        if seqs < 1:
            continue
        tokens = max(most, min(seqs, ((1 << 24) - 1) // (heads * group)))
        if tokens * heads * group >= 1 << 24:
            continue
        s = _shape(head_dim=dim, num_kv_heads=heads)
        m, c = pb.make_model(s), pb.PkvPagedCache(tag=tag)
        window = int(rng.choice([0, 100]))
        b = pb.PkvBatch(num_seqs=seqs, num_tokens=tokens, max_tokens=most, pages_per_seq=int(2 ** rng.uniform(0, 13)))
        a = pb.PkvAttention(num_q_heads=heads * group, window=window, scale=0.1)
        out = ctypes.c_uint64()
        st = lib.pkv_attention_workspace(ctypes.byref(m), ctypes.byref(c), ctypes.byref(b), ctypes.byref(a),
                                         ctypes.byref(out))
        assert st == OK, (dim, tag, heads, group, most, seqs, tokens)
        taken += 1
    assert taken > 1000


@pytest.mark.parametrize("heads,group,tag,seqs,tokens,most", [(16, 33, 3, 390000, 1000, 1), (8, 1, 3, 900000, 900000, 48)])
def test_launches_of_more_workgroups_are_refused(heads, group, tag, seqs, tokens, most):
    """Three shares of rows, and pieces for half as many sequences again: past 2^24 workgroups at 256 channels."""
    s = _shape(head_dim=256, num_kv_heads=heads)
    m, c = pb.make_model(s), pb.PkvPagedCache(tag=tag)
    b = pb.PkvBatch(num_seqs=seqs, num_tokens=tokens, max_tokens=most, pages_per_seq=1000)
    with pytest.raises(pb.PkvError) as e:
        pb.pkv_attention_workspace(m, c, b, pb.PkvAttention(num_q_heads=heads * group, scale=0.1))
    assert e.value.status == BAD


@pytest.mark.parametrize("dtype,held,ok", [
    ("float16", "float16", True), ("bfloat16", "bfloat16", True), ("float16", "int16", True), ("bfloat16", "int16", True),
    ("bfloat16", "uint16", True), ("float16", "bfloat16", False), ("bfloat16", "float16", False),
    ("bfloat16", "float32", False), ("float16", "int8", False)])
@pytest.mark.parametrize("which", ["both", "v"])
def test_a_16_bit_cache_holds_its_own_type_or_bits(dtype, held, ok, which):
    """Floating caches of the other 16-bit type would be read as this one; bits (as device.alloc_caches makes them) pass,
    here as far as the refusal of host memory."""
    torch = pytest.importorskip("torch")
    from paper_2609_26219_amd import serving

    of = lambda name: torch.zeros((2, 3, 16, 2, 64), dtype=getattr(torch, name))  # noqa: E731
    with pytest.raises(ValueError, match="device memory" if ok else "hold"):
        serving.PagedCache(2, 64, 16, getattr(torch, dtype), 0, k_cache=of(held if which == "both" else dtype),
                           v_cache=of(held))


def test_rows_of_a_sequence_stay_within_the_call(tmp_path):
    """The kernels' clamps of what the host cannot see, compiled for the host (serve_rows_check.cpp)."""
    import os
    import shutil
    import subprocess

    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    here = os.path.dirname(os.path.abspath(__file__))
    root, exe = os.path.dirname(here), str(tmp_path / "check")
    subprocess.run([cxx, "-O1", "-fwrapv", "-std=c++17", "-Wall", "-Wextra", "-I", os.path.join(root, "include"),
                    "-I", os.path.join(root, "paper_2609_26219_amd", "csrc"), os.path.join(here, "serve_rows_check.cpp"),
                    "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout + run.stderr
