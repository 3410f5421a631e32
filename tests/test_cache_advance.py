"""PagedKVCache.advance: how long the counts on the device live, without a GPU: its tensors
replaced by ones that note what is done with them."""
from contextlib import contextmanager

import pytest
import torch

from paper_2607_22586_gb300.cache import PagedKVCache


class _Lens:
    is_cuda = True

    def add_(self, counts):
        self.last = counts


class _Counts:
    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream)


@pytest.fixture
def cache(monkeypatch):
    c = PagedKVCache(6, 2, 64, torch.bfloat16, batch=2, rows=32, page_size=16, device="cpu")
    c.lens, c.state = _Lens(), {"device": 0, "capturing": {1: False}, "stream": "s0"}
    c._counts = {(2, 3): _Counts()}

    @contextmanager
    def on_device(self):
        old, c.state["device"] = c.state["device"], 1
        yield
        c.state["device"] = old

    monkeypatch.setattr(PagedKVCache, "_on_device", on_device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: c.state["capturing"].get(c.state["device"], False))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: (c.state["device"], c.state["stream"]))
    return c


def test_counts_outlive_their_use_on_another_stream(cache):
    """They may be dropped while a stream other than the one they were made on still reads them."""
    counts = cache._counts[2, 3]
    cache.advance([2, 3])
    assert cache.lens.last is counts and counts.streams == [(1, "s0")]
    cache.state["stream"] = "s1"
    cache.advance([2, 3])
    assert counts.streams[-1] == (1, "s1") and not cache._captured


def test_captured_counts_are_kept_whatever_device_is_current(cache):
    cache.state["capturing"][1] = True
    cache.advance([2, 3])
    assert cache._captured == [cache._counts[2, 3]]
    cache.state["capturing"] = {0: True, 1: False}     # another device's stream is being captured
    cache.advance([2, 3])
    assert len(cache._captured) == 1


def test_equal_counts_need_no_tensor(cache):
    cache.advance([4, 4])
    assert cache.lens.last == 4
