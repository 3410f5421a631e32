"""Which indices and counts PagedKVCache.fill hands on: without a GPU, the entry points
replaced by ones that note their arguments."""
from contextlib import nullcontext

import pytest
import torch

from paper_2607_22586_gb300 import _lib as L
from paper_2607_22586_gb300.cache import PagedKVCache
from paper_2607_22586_gb300.selector import KVSelector


@pytest.fixture
def filled(monkeypatch):
    """A selector, a cache, and what the last fill was given: (idx, counts)."""
    seen = {}

    def fill(shape, cache, K, V, idx, count, ws, n, stream=None):
        seen["got"] = (idx, count)
        return 0

    monkeypatch.setattr(L, "mmshift_cache_fill", fill)
    monkeypatch.setattr(L, "mmshift_select", lambda *a: 0)
    monkeypatch.setattr(L, "mmshift_select_with_stats", lambda *a: 0)
    monkeypatch.setattr(L, "mmshift_select_head_budgets", lambda *a: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: 0)
    monkeypatch.setattr(PagedKVCache, "_on_device", lambda self: nullcontext())
    sel = KVSelector(6, 2, 64, 8, torch.bfloat16, [0, 40], [10], n_layers=2, params=L.default_params(n_proxies=32, n_groups=2),
                     device="cpu")
    cache = PagedKVCache(6, 2, 64, torch.bfloat16, batch=1, rows=32, n_layers=2, page_size=16, device="cpu")
    K = torch.zeros((2, 40, 2, 64), dtype=torch.bfloat16)
    Q = torch.zeros((2, 1, 8, 6, 64), dtype=torch.bfloat16)
    return sel, cache, K, Q, seen


def test_counts_without_indices_are_used(filled):
    sel, cache, K, Q, seen = filled
    counts = torch.ones((2, 1, 2), dtype=torch.int32)
    sel(K, K, Q)
    cache.fill(sel, K, K, counts=counts)
    assert seen["got"][0] is sel.out_idx and seen["got"][1] is counts
    sel(K, K, Q, head_budgets=counts)
    cache.fill(sel, K, K, counts=counts)
    assert seen["got"][1] is counts and sel.out_count is not counts


def test_indices_come_without_the_selection_s_counts(filled):
    sel, cache, K, Q, seen = filled
    idx, counts = sel.out_idx.clone(), torch.ones((2, 1, 2), dtype=torch.int32)
    sel(K, K, Q, head_budgets=counts)
    cache.fill(sel, K, K, idx)
    assert seen["got"][0] is idx and seen["got"][1] is None
    cache.fill(sel, K, K, idx, counts)
    assert seen["got"][0] is idx and seen["got"][1] is counts
    cache.fill(sel, K, K)
    assert seen["got"][0] is sel.out_idx and seen["got"][1] is sel.out_count


def test_counts_of_an_earlier_selection_are_not_used(filled):
    """A selection without budgets per head keeps every head's budget, whatever one before it kept."""
    sel, cache, K, Q, seen = filled
    budgets = torch.ones((2, 1, 2), dtype=torch.int32)
    stats = torch.zeros((2, 1, 2, 6 * 64))
    for again in ({}, {"stats": stats}):
        sel(K, K, Q, head_budgets=budgets)
        cache.fill(sel, K, K)
        assert seen["got"][1] is sel.out_count
        kept = sel.out_count
        sel(K, K, Q, **again)
        cache.fill(sel, K, K)
        assert seen["got"][1] is None and sel.out_count is kept
