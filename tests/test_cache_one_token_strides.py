"""PagedKVCache takes rows whose strides differ only along axes of one element: without a
GPU, the entry points replaced by ones that note their arguments."""
from contextlib import nullcontext

import pytest
import torch

from paper_2607_22586_gb300 import _lib as L
from paper_2607_22586_gb300.cache import PagedKVCache


@pytest.fixture
def call(monkeypatch):
    got = {}

    def append(shape, cache, K, V, stride, ws, n, stream=None):
        got.update(stride=stride, layers=shape.n_layers, layer_stride=shape.layer_stride_kv)
        return 0

    monkeypatch.setattr(L, "mmshift_cache_append", append)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: 0)
    monkeypatch.setattr(PagedKVCache, "_on_device", lambda self: nullcontext())

    def make(layers):
        return PagedKVCache(6, 2, 64, torch.bfloat16, batch=1, rows=32, n_layers=layers, page_size=16, device="cpu"), got

    return make


def _projected(*shape):
    """Rows inside wider ones."""
    return torch.zeros((*shape[:-2], 10, 64), dtype=torch.bfloat16)[..., 6:8, :]


def test_one_token(call):
    """One token's K, made anew (rotated), and its V, a view of a projection's output."""
    cache, got = call(2)
    k, v = torch.zeros((1, 2, 64), dtype=torch.bfloat16), _projected(1, 2, 64)
    assert k.stride() != v.stride()
    cache.append(k, v, [1], layer=0)
    assert got["stride"] >= 128 and got["layers"] == 1
    # all layers: they are equally far apart, whatever the one token's stride says
    k, v = _projected(2, 1, 2, 64), torch.zeros((2, 640), dtype=torch.bfloat16).as_strided((2, 1, 2, 64), (640, 128, 64, 1))
    assert k.stride(0) == v.stride(0) and k.stride(1) != v.stride(1)
    cache.append(k, v, [1])
    assert got["stride"] >= 128 and got["layer_stride"] == 640


def test_one_layer(call):
    cache, got = call(1)
    k = torch.zeros((3, 3, 2, 64), dtype=torch.bfloat16)
    cache.append(k[:1], k.transpose(0, 1)[:1].contiguous().as_strided((1, 3, 2, 64), (7, 128, 64, 1)), [3])
    assert got["stride"] == 128


def test_several_tokens_or_layers_still_have_to_agree(call):
    cache, _ = call(2)
    k, v = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16), _projected(2, 3, 2, 64)
    for args in ((k, v, [3]), (k[0], v[0], [3], 0), (k[:, :1].contiguous(), _projected(2, 1, 2, 64), [1])):
        with pytest.raises(ValueError):
            cache.append(*args)
