"""The example runs, from a checkpoint to decoded tokens."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny", "llama8b_1l"])
def test_resume_and_decode(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "resume_and_decode.py")
    spec = importlib.util.spec_from_file_location("resume_and_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(name, steps=5, window=100)
    assert got["repaired_rows"] > 0 and got["repaired_finite"] and got["replays_agree"] and got["decoded"] == 5
    # Values are drawn with a spread near 1 (the checkpoint's with a few channels 8 times that): 16 codes over a row's
    # range are off by up to a fifteenth of it, and so is an average of them.
    assert 0.0 < got["worst_difference"] < 8.0


def test_every_attention_of_the_example_against_the_oracle(monkeypatch):
    """Each eager attention of the tiny example, and what its last replay left, against fp64 attention over the caches as
    they lie; and the 4-bit cache's rows within half a step of the 16-bit ones they came from."""
    import numpy as np
    import torch

    from oracle import serving as os_
    from serving_cases import Case, check_attention

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "resume_and_decode.py")
    spec = importlib.util.spec_from_file_location("resume_and_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    host = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    attention, calls, rows_of = example.serving.attention, [], {}

    def as_case(cache, batch, q):
        case = Case.__new__(Case)
        case.tag, case.dtype, case.D, case.P, case.H = (cache.tag, int(cache.dtype == torch.bfloat16), cache.head_dim,
                                                        cache.page_size, cache.num_kv_heads)
        start, lens, table, positions = batch.keep
        case.start, case.lens, case.table = (t.cpu().numpy() for t in (start, lens, table))
        case.positions = None if positions is None else positions.cpu().numpy()
        case.pool, case.tokens, case.most_kv = cache.pool_pages, batch.num_tokens, int(case.lens.max())
        case.q = host(q)
        if cache.tag == 0:
            layer = lambda t: host(t[0] if t.dim() == 5 else t)  # noqa: E731
            case.cache = {"kv": [layer(cache.k_cache), layer(cache.v_cache)]}
        else:
            case.cache = {"codes": cache.codes.reshape(cache.codes.shape[-3:]).cpu().numpy(),
                          "scales": host(cache.scales).reshape(cache.scales.shape[-5:])}
        return case

    def checked(cache, batch, q, window=0, sinks=0, out=None, return_lse=False, **kw):
        got = attention(cache, batch, q, window=window, sinks=sinks, out=out, return_lse=return_lse, **kw)
        if torch.cuda.is_current_stream_capturing():
            return got
        case = as_case(cache, batch, q)
        o = got[0] if return_lse else got
        lse = got[1].cpu().numpy() if return_lse else case.attend(None, window, sinks)[1].astype(np.float32)
        check_attention(case, host(o), lse, window, sinks)
        calls.append((cache.tag, bool(window), case.tokens))
        if case.tokens == 1:
            rows_of[cache.tag] = case
        return got

    monkeypatch.setattr(example.serving, "attention", checked)
    got = example.run("tiny", steps=3, window=20, sinks=2)
    assert got["replays_agree"]  # the replays with the eager windowed calls, which were checked
    steps = [c for c in calls if c[2] == 1]
    assert calls[0] == (0, False, got["repaired_rows"])
    assert steps.count((0, False, 1)) == steps.count((3, False, 1)) == 3 and steps.count((3, True, 1)) == 4
    sixteen, four = rows_of[0], rows_of[3]
    n = int(sixteen.lens[0])
    assert n == int(four.lens[0]) == got["context"] + 3
    for t in range(n):
        for which in range(2):
            for h in range(sixteen.H):
                x, y = (os_.row(c.cache, c.tag, c.P, c.dtype, which, int(c.table[0, t // c.P]), t % c.P, h)[0]
                        for c in (sixteen, four))
                scale = float(four.cache["scales"][int(four.table[0, t // four.P]), h, which, t % four.P, 0:1]
                              .view(np.float16)[0])
                assert np.abs(x - y).max() <= scale / 2 * (1 + 2.0 ** -20)
