"""Several host threads on one paged cache, without a GPU: the library's calls are replaced by functions that note what
they were given and hold a thread where another one can get in between.

A cache lies in host memory here and says that it is on a device."""
import threading

import pytest
import torch

from paper_2609_26219_amd import binding as pb
from paper_2609_26219_amd import serving
from paper_2609_26219_amd import workloads as wl

WAIT = 20.0  # seconds before a test gives up on a thread


class Elsewhere(torch.Tensor):
    @property
    def device(self):
        return torch.device("cuda", 0)


def _zeros(shape, dtype):
    return torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)


def _cache(layers=3):
    codes, scales = _zeros((layers, 4, 2, 16 * 64), torch.uint8), _zeros((layers, 4, 2, 2, 16, 2), torch.float16)
    return serving.PagedCache(2, 64, 16, torch.bfloat16, wl.TAG_K4V4, codes=codes, scales=scales)


def _batch(rows):
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return serving.Batch(ints(0, rows), ints(40), ints(0, 1, 2).view(1, 3), rows)


def _rows(heads, n=1):
    return torch.zeros((n, heads, 64), dtype=torch.bfloat16)


class Thread(threading.Thread):
    """A thread whose error is raised by join."""

    def __init__(self, work):
        super().__init__(daemon=True)
        self.work, self.error = work, None

    def run(self):
        try:
            self.work()
        except BaseException as e:  # noqa: BLE001
            self.error = e

    def join(self, timeout=WAIT):
        super().join(timeout)
        assert not self.is_alive()
        if self.error:
            raise self.error


@pytest.fixture
def one_stream(monkeypatch):
    monkeypatch.setattr(serving, "_stream", lambda cache: 7)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)


@pytest.mark.parametrize("other", ["append", "read", "attention"])
def test_a_call_keeps_its_layer_while_another_thread_calls(monkeypatch, one_stream, other):
    """Attention of layer 0 is held between its workspace query and its launch, while a call of layer 2 runs whole."""
    cache, batch = _cache(), _batch(1)
    inside, go, seen = threading.Event(), threading.Event(), []

    def workspace(model, struct, b, a):
        if not inside.is_set():
            inside.set()
            assert go.wait(WAIT)
        return 0

    def launched(model, struct, *rest):
        seen.append(struct.layer)
        return pb.PKV_OK

    monkeypatch.setattr(pb, "pkv_attention_workspace", workspace)
    for name in ("pkv_attention_status", "pkv_cache_append_status", "pkv_cache_read_status"):
        monkeypatch.setattr(pb, name, launched)
    first = Thread(lambda: serving.attention(cache, batch, _rows(4), layer=0))
    first.start()
    assert inside.wait(WAIT)
    calls = {"append": lambda: serving.append(cache, batch, _rows(2), _rows(2), layer=2),
             "read": lambda: serving.read(cache, batch, layer=2, out=(_rows(2), _rows(2))),
             "attention": lambda: serving.attention(cache, batch, _rows(4), layer=2)}
    calls[other]()
    go.set()
    first.join()
    assert seen == [2, 0]


def test_a_layer_that_is_not_there_is_the_librarys_to_refuse(one_stream):
    cache, batch = _cache(), _batch(1)
    for layer in (-1, 3, 1 << 20):
        for call in (lambda: serving.append(cache, batch, _rows(2), _rows(2), layer=layer),
                     lambda: serving.attention(cache, batch, _rows(4), layer=layer)):
            with pytest.raises(pb.PkvError) as e:
                call()
            assert e.value.status == pb.PKV_ERR_INVALID_ARGUMENT


def test_calls_that_share_scratch_memory_are_enqueued_one_after_the_other(monkeypatch, one_stream):
    """Two threads on one stream use the same scratch memory, so the kernels of one call (attention, then the join of its
    parts) have to be enqueued with none of the other's between them, and the memory has to stay the call's until then,
    also where the other call wants more of it."""
    cache, batch = _cache(), _batch(1)
    sizes = {"first": 1 << 10, "second": 1 << 20}
    inside, waiting, log = threading.Event(), threading.Event(), []

    def workspace(model, struct, b, a):
        return sizes[threading.current_thread().name]

    def launched(model, struct, b, a, stream):
        name = threading.current_thread().name
        log.append((name, "begins"))
        if name == "first":
            inside.set()
            waiting.wait(1.0)  # the second thread, if nothing holds it, is in here within that time
            held = cache._workspace[stream]
            assert held[1] == a.workspace and held[0] >= a.workspace_bytes
        else:
            waiting.set()
        log.append((name, "ends"))
        return pb.PKV_OK

    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(pb, "pkv_attention_workspace", workspace)
    monkeypatch.setattr(pb, "pkv_attention_status", launched)
    threads = [Thread(lambda: serving.attention(cache, batch, _rows(4))) for _ in range(2)]
    for t, name in zip(threads, sizes):
        t.name = name
    threads[0].start()
    assert inside.wait(WAIT)
    threads[1].start()
    for t in threads:
        t.join()
    assert log == [("first", "begins"), ("first", "ends"), ("second", "begins"), ("second", "ends")]


def test_scratch_memory_is_free_again_after_a_refused_call(monkeypatch, one_stream):
    cache, batch = _cache(), _batch(1)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(pb, "pkv_attention_workspace", lambda *a: 64)
    monkeypatch.setattr(pb, "pkv_attention_status", lambda *a: pb.PKV_ERR_DEVICE)
    with pytest.raises(pb.PkvError):
        serving.attention(cache, batch, _rows(4))
    monkeypatch.setattr(pb, "pkv_attention_status", lambda *a: pb.PKV_OK)
    again = Thread(lambda: serving.attention(cache, batch, _rows(4)))
    again.start()
    again.join()


def test_numbers_past_32_bits_do_not_wrap(monkeypatch, one_stream):
    """A layer past 32 bits is refused as any other that is not there; a window or sinks past them cover everything."""
    cache, batch = _cache(), _batch(1)
    for layer in (1 << 32, -(1 << 32), (1 << 32) + 1):
        with pytest.raises(pb.PkvError) as e:
            serving.append(cache, batch, _rows(2), _rows(2), layer=layer)
        assert e.value.status == pb.PKV_ERR_INVALID_ARGUMENT
    for past in (1 << 31, 1 << 32, (1 << 32) + 4, 1 << 70):
        for kw in (dict(window=-past), dict(window=1 - past), dict(sinks=-past)):
            with pytest.raises(pb.PkvError) as e:
                serving.attention(cache, batch, _rows(4), **kw)
            assert e.value.status == pb.PKV_ERR_INVALID_ARGUMENT
    seen = []
    monkeypatch.setattr(pb, "pkv_attention_workspace", lambda *a: 0)
    monkeypatch.setattr(pb, "pkv_attention_status", lambda m, c, b, a, s: seen.append((a.window, a.sinks)) or pb.PKV_OK)
    for past in (1 << 31, 1 << 32, (1 << 32) + 4, 1 << 70):
        serving.attention(cache, batch, _rows(4), window=past, sinks=past)
        serving.attention(cache, batch, _rows(4), window=7, sinks=2)
    assert set(seen) == {(2 ** 31 - 1, 2 ** 31 - 1), (7, 2)}
