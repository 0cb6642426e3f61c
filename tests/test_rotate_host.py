"""Host half of the rotating calls, without a GPU: refusals before any HIP call, and the kernels' sine and cosine, compiled
for the host, against long double ones."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from paper_2609_26219_amd import binding as pb
from paper_2609_26219_amd import build as pkv_build
from test_serving_host import A, BAD, OK, TAG, _gpu_present, _shape


def _call(which="rotate", shape=None, batch=None, rotation=None, rows=None, cache=None):
    s = shape or _shape()
    m = pb.make_model(s)
    b = dict(num_seqs=2, num_tokens=0, max_tokens=0, pages_per_seq=4, max_kv_len=0, token_start=A, kv_lens=A,
             positions=None, page_table=A)
    b.update(batch or {})
    r = dict(num_heads=8, amplitude=1.0, position_offset=None, x=A, x_token_stride=1024, x_head_stride=128, out=2 * A,
             out_token_stride=1024, out_head_stride=128)
    r.update(rotation or {})
    b, r = pb.PkvBatch(**b), pb.PkvRotation(**r)
    if which == "rotate":
        return pb.pkv_rotate_status(m, b, r)
    cb, sb = pb.pkv_cache_size(s, 3)
    c = dict(tag=3, layer=1, codes=A, code_bytes=cb, scales=A, scale_bytes=sb)
    c.update(cache or {})
    k = dict(k=A, v=A, token_stride=512, head_stride=128)
    k.update(rows or {})
    return pb.pkv_cache_append_rotated_status(m, pb.PkvPagedCache(**c), b, k["k"], k["v"], k["token_stride"],
                                              k["head_stride"], r)


BOTH = pytest.mark.parametrize("which", ["rotate", "append"])


@BOTH
def test_nothing_to_do_is_ok(which):
    assert _call(which) == OK
    assert _call(which, batch=dict(num_seqs=0, num_tokens=5)) == OK
    if which == "rotate":
        assert _call(which, batch=dict(num_tokens=5), rotation=dict(num_heads=0, x=None, out=None)) == OK


@BOTH
@pytest.mark.parametrize("rotation", [dict(num_heads=-1), dict(amplitude=float("nan")), dict(amplitude=float("inf")),
                                      dict(position_offset=A + 2), dict(x=None), dict(out=None), dict(x=A + 8),
                                      dict(out=A + 2), dict(x_token_stride=4), dict(x_head_stride=64),
                                      dict(out_head_stride=120), dict(out_token_stride=-8),
                                      dict(out=A, out_token_stride=2048), dict(num_heads=1 << 30)])
def test_rotation_refusals(which, rotation):
    assert _call(which, batch=dict(num_tokens=3), rotation=rotation) == BAD


@BOTH
@pytest.mark.parametrize("batch", [dict(num_seqs=-1), dict(num_tokens=-1), dict(pages_per_seq=0), dict(max_kv_len=-1),
                                   dict(num_tokens=1 << 28), dict(num_tokens=3, token_start=None),
                                   dict(num_tokens=3, kv_lens=A + 2), dict(num_tokens=3, positions=A + 1)])
def test_batch_refusals(which, batch):
    assert _call(which, batch=batch) == BAD


def test_append_refusals():
    assert _call("append", cache=dict(tag=4)) == TAG
    assert _call("append", cache=dict(layer=2)) == BAD
    for rows in (dict(k=None), dict(v=A + 2), dict(token_stride=4), dict(head_stride=64)):
        assert _call("append", batch=dict(num_tokens=1), rows=rows) == BAD


def test_null_structures():
    lib, m, b = pb.load(), pb.make_model(_shape()), pb.PkvBatch(num_seqs=1, pages_per_seq=4)
    r = pb.PkvRotation(num_heads=0, amplitude=1.0)
    ref = ctypes.byref
    assert lib.pkv_rotate(None, ref(b), ref(r), None) == BAD
    assert lib.pkv_rotate(ref(m), None, ref(r), None) == BAD
    assert lib.pkv_rotate(ref(m), ref(b), None, None) == BAD
    c = pb.PkvPagedCache(tag=3)
    assert lib.pkv_cache_append_rotated(ref(m), ref(c), ref(b), None, None, 512, 128, None, None) == BAD


def test_models_with_bad_rope_are_refused():
    for kw in (dict(rope_style=3), dict(rotary_dim=24), dict(inv_freq=(float("nan"),) * 64)):
        assert _call(shape=_shape(**kw)) == BAD


def test_sine_and_cosine(tmp_path):
    """Within 2^-52 of long double ones, up to the angles of far positions and at multiples of pi / 2."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    with open(os.path.join(pkv_build.CSRC, "serve.hip")) as f:
        body = re.search(r"__device__ __forceinline__ (void sine_cosine\(.*?\n})", f.read(), re.S).group(1)
    src = tmp_path / "sine.cpp"
    src.write_text('extern "C" ' + body.replace("void sine_cosine", "void sine_cosine", 1) + "\n")
    lib = str(tmp_path / "libsine.so")
    subprocess.run([cxx, "-O1", "-std=c++17", "-mfma", "-shared", "-fPIC", str(src), "-o", lib], check=True)
    fn = ctypes.CDLL(lib).sine_cosine
    fn.argtypes = [ctypes.c_double, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    rng = np.random.default_rng(0)
    angles = np.concatenate([rng.uniform(-10, 10, 2000), 10.0 ** rng.uniform(-12, 9.3, 6000), [0.0, -0.0],
                             np.arange(-40, 400) * (np.pi / 4), np.arange(1 << 20, (1 << 20) + 500) * (np.pi / 2),
                             np.nextafter(np.arange(1, 200) * (np.pi / 4), 0), -10.0 ** rng.uniform(-3, 9.3, 2000)])
    s, c = ctypes.c_double(), ctypes.c_double()
    for a in angles:
        fn(a, s, c)
        want = np.longdouble(a)
        assert abs(np.longdouble(s.value) - np.sin(want)) <= 2.0 ** -52 and \
            abs(np.longdouble(c.value) - np.cos(want)) <= 2.0 ** -52, a


@BOTH
def test_heads_that_a_workgroup_can_count(which):
    """A workgroup goes over a token's heads in steps, whose count stays within 32 bits up to 2^30 heads."""
    for heads in ((1 << 30) + 1, (1 << 31) - 1):
        assert _call(which, batch=dict(num_tokens=1), rotation=dict(num_heads=heads)) == BAD
    if not _gpu_present():  # (past every check, and no device)
        assert _call(which, batch=dict(num_tokens=1), rotation=dict(num_heads=1 << 30)) == pb.PKV_ERR_DEVICE


@pytest.mark.skipif(_gpu_present(), reason="with a GPU these addresses are no device memory")
def test_the_page_table_of_a_rotation_is_not_read():
    for table in (None, A + 2):
        assert _call(batch=dict(num_tokens=3, page_table=table)) == pb.PKV_ERR_DEVICE  # (past every check, and no device)
        assert _call("append", batch=dict(num_tokens=3, page_table=table)) == BAD
    assert _call("append", batch=dict(num_tokens=3)) == pb.PKV_ERR_DEVICE
